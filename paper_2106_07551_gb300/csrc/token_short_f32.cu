// Short rows of fp32 logits.
#include "token_short.cuh"

namespace malib {

cudaError_t launch_token_short_f32(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    return launch_short_type<float>(a, op, n_sm, s);
}

}  // namespace malib
