// Long rows of f16 logits.
#include "token_ring.cuh"

namespace malib {

cudaError_t launch_token_ring_f16(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    return launch_ring_type<__half>(a, op, n_sm, s);
}

}  // namespace malib
