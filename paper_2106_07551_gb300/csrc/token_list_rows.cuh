// Lists and draws: the kernel that takes rows of a length, number and list.
#pragma once

#include "token_list.cuh"
#include "token_list_tiny.cuh"

namespace malib {

namespace {

template <class T, int kOp>
cudaError_t launch_list_op(const ListArgs& a, int n_sm, cudaStream_t s) {
    if (a.V <= 8) return launch_list_tiny<T, kOp, 8>(a, n_sm, s);
    if (a.V <= 16) return launch_list_tiny<T, kOp, 16>(a, n_sm, s);
    if constexpr (kOp == kListDrawAll) {
        if (a.V <= 32) return launch_list_tiny<T, kOp, 32>(a, n_sm, s);
    }
    const int64_t nv = (a.V + 2 * (int64_t)Elt<T>::W - 2) / Elt<T>::W;               // most vectors of a row
    ListShape sh{1, (int)nv, -1, 0, 0};
    // Clusters while the CTAs' lists can be sorted together.
    for (int c = 2; c <= 8 && (nv + c - 1) / c >= 512; c *= 2)
        if (a.n * c <= 4 * (int64_t)n_sm && (int64_t)c * a.K <= kListCap / 2) {
            sh.cluster = c;
            sh.slice = (int)((nv + c - 1) / c);
        }
    if (sh.slice <= 256) return launch_list_threads<T, kOp, 32>(a, sh, s);
    if (sh.cluster == 1 && sh.slice <= kManyBatches * 128 * kListPer) return launch_list_threads<T, kOp, 128>(a, sh, s);
    return launch_list_threads<T, kOp, 256>(a, sh, s);
}

template <class T>
cudaError_t launch_list_type(const ListArgs& a, int op, int n_sm, cudaStream_t s) {
    if (op == kListTop) return launch_list_op<T, kListTop>(a, n_sm, s);
    if (op == kListDraw) return launch_list_op<T, kListDraw>(a, n_sm, s);
    return launch_list_op<T, kListDrawAll>(a, n_sm, s);
}

}  // namespace

}  // namespace malib
