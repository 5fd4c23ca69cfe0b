// Long rows of fp32 logits.
#include "token_ring.cuh"

namespace malib {

cudaError_t launch_token_ring_f32(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    return launch_ring_type<float>(a, op, n_sm, s);
}

}  // namespace malib
