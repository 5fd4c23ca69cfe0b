// The most likely entries and the draw of fp16 logits.
#include "token_list_rows.cuh"

namespace malib {

cudaError_t launch_token_list_f16(const ListArgs& a, int op, int n_sm, cudaStream_t s) {
    return launch_list_type<__half>(a, op, n_sm, s);
}

}  // namespace malib
