// Sixteen bytes from an address that is not a multiple of 16, in two aligned loads: rows
// of logits and gradient that are not aligned alike.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace malib {

template <int kWord>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, uint32_t bits) {
    const uint32_t w[9] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, 0};
    return make_uint4(__funnelshift_r(w[kWord], w[kWord + 1], bits), __funnelshift_r(w[kWord + 1], w[kWord + 2], bits),
                      __funnelshift_r(w[kWord + 2], w[kWord + 3], bits),
                      __funnelshift_r(w[kWord + 3], w[kWord + 4], bits));
}
__device__ __forceinline__ uint4 load_shifted(const uint8_t* p, int by) {   // p: 16-byte aligned, 0 < by < 16
    const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 16);
    const uint32_t bits = 8u * (by & 3);
    switch (by >> 2) {
        case 0: return shifted<0>(a, b, bits);
        case 1: return shifted<1>(a, b, bits);
        case 2: return shifted<2>(a, b, bits);
        default: return shifted<3>(a, b, bits);
    }
}

}  // namespace malib
