// Lists and draws: the kernel that takes rows of a length, number and list.
#pragma once

#include "token_draw_stream.cuh"
#include "token_list.cuh"
#include "token_list_short.cuh"
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
    if (nv <= 256) return launch_list_short<T, kOp>(a, nv, n_sm, s);
    ListShape sh{};
    sh.cluster = 1;
    sh.group_log = -1;
    // CTAs a row: as many as there are SMs for twice, with slices of 24 KB or more. us, C = 1, 2, 4 and 8:
    // lists of 20 from one row of 131,072 bf16 entries 18.5, 15.4, 13.6, 14.6, of 64 from 100 rows 20, 21,
    // 31, 36; of 5 from 61 x 50,001 fp16 12.9, 11.3, 12.8, 16.5; draws from one row of a million 76, 35,
    // 21, 15. Slices of 128 KB or more, by 2 or 3 up to 13 CTAs for 4 SMs (of the 16 that lists hold, and the 12
    // of draws): of 1 from 184,696 fp32, C = 1, 2 and 3, 164 rows 60, 43, 35, 200 rows 62, 43, 51, 240 rows 62, 46, 57; of
    // 10 from 250,000 bf16, 164 rows 52, 38, 32, 200 rows 54, 39, 48, 240 rows 54, 41, 54. (At 300 rows, which the next
    // rule takes, 64, 50, 61 and 54, 42, 58: 2 would be best.) Rows whose sums would need their roundings' errors, by 3
    // up to 7 CTAs an SM, which are 354 rows: of 64 from 140,001 fp32, C = 1, 2 and 3, 354 rows 65, 67, 58, 420 rows
    // 67, 73, 76, from 200,001 87, 91, 77 and 88, 97, 100. Long lists, whose selection takes as long as the sums, from
    // rows of more than 288 KB, also over several rounds, by 2 or 3: of 1,024 from 333 x 151,111 fp32, C = 1, 2, 3 and
    // 4, 131, 109, 86, 94, 1,000 rows 251, 238, 223, 225; of 300 from 80,001, C = 1, 2 and 3, 333 rows 66, 53, 51, 811
    // 108, 90, 106, 1,300 165, 137, 159, from 160,001 bf16 79, 66, 63, 129, 110, 136, 195, 171, 205.
    for (int c = 2; c <= 8; c += c == 2 ? 1 : c == 3 ? 1 : c) {
        const int64_t slice = (nv + c - 1) / c;
        if ((slice >= 1536 && c != 3 && a.n * c <= 2 * (int64_t)n_sm) ||
            (slice >= 8192 && c <= 3 && a.n * c * 4 <= (kOp == kListDrawAll ? 12 : 13) * (int64_t)n_sm) ||
            (a.K > 0 && c == 3 && nv > kManyBatches * 256 * kListPer && a.n * c <= 7 * (int64_t)n_sm) ||
            (a.K > 128 && slice >= 9216 && c <= 3 && a.n * c <= 16 * (int64_t)n_sm))
            sh.cluster = c;
    }
    // What the CTAs list is sorted together: K entries each as long as that is little, else a share of K with
    // a quarter more, which has them all unless a slice has more than its share.
    sh.slice = (int)((nv + sh.cluster - 1) / sh.cluster);
    if (kOp == kListDrawAll) sh.slice = (sh.slice + 256 * kListPer - 1) / (256 * kListPer) * (256 * kListPer);    // whole batches
    sh.slice_K = sh.cluster * a.K <= kListCap / 2 ? a.K : a.K / sh.cluster * 5 / 4 + 32;
    if constexpr (kOp == kListDrawAll) {
        if (sh.cluster == 1 && nv <= kStreamMostBatches * kStreamBatch) return launch_draw_stream<T>(a, nv, n_sm, s);
    }
    // Rows that 128 threads sweep in one batch or two: a row's selection is a chain of short steps, and more of them
    // go on at a time by blocks of 64. us, 128 and 64 threads: lists of 64 from 8,192 rows of 3,000 bf16 entries
    // 71 and 54, of 10 from 12,000 69 and 56, of 64 from 16,384 84 and 87, of 256 from 3,000 133 and 178.
    if constexpr (kOp != kListDrawAll) {
        if (sh.cluster == 1 && sh.slice <= 1536 && a.K <= 128) return launch_list_threads<T, kOp, 64>(a, sh, s);
        if (sh.cluster == 1 && sh.slice <= kManyBatches * 128 * kListPer) return launch_list_threads<T, kOp, 128>(a, sh, s);
    }
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
