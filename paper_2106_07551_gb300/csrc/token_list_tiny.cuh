// Lists and draws of rows of up to N entries (the actions of the environments): a thread a row, its entries in
// registers. An entry's place in the order is how many come before it, and the mass before it is theirs.
// Rows that follow one another without a gap go through shared memory, so that neighbouring threads
// read neighbouring entries.
// 102,400 draws from 15 fp32 actions: 8.8 us on the device (latency: issue slots 32 %), by a warp a row 105.
#pragma once

#include "token_list.cuh"

namespace malib {

namespace {

constexpr int kTinyThreads = 128;

template <class T, int kOp, int N>
__global__ void __launch_bounds__(kTinyThreads) token_list_tiny_kernel(ListArgs a) {
    __shared__ T tile[kTinyThreads * N];
    const int tid = threadIdx.x;
    const bool flat = a.ld == a.V;
    wait_for_previous();
    let_next_start();
    for (int64_t row0 = (int64_t)blockIdx.x * kTinyThreads; row0 < a.n; row0 += (int64_t)gridDim.x * kTinyThreads) {
        const int rows = (int)min((int64_t)kTinyThreads, a.n - row0), entries = rows * a.V;
        const bool in_range = tid < rows;
        const int64_t row = row0 + (in_range ? tid : 0);
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        if (flat) {
            const T* first = static_cast<const T*>(a.z) + row0 * a.V;
            for (int e = tid; e < entries; e += kTinyThreads) tile[e] = first[e];
        }
        const int token = a.tokens ? a.tokens[row] : 0;
        bool live = in_range && token >= 0;
        if (kOp == kListTop && token >= a.V) {
            if (in_range) atomicOr(a.err, ERRBIT_BAD_TOKEN);
            live = false;
        }
        float u = 0.f;
        if (kOp != kListTop && live) u = row_uniform(a, row);
        float v[N];
        if (flat) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = j < a.V ? Elt<T>::get(tile[tid * a.V + j]) : -INFINITY;
            __syncthreads();
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = j < a.V ? Elt<T>::get(z[j]) : -INFINITY;
        }
        if (!in_range) continue;
        RowStat r{v[0], 0.f, 0.f};
        float zt = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            r.m = max_nan(r.m, v[j]);
            if (kOp == kListTop && j == token) zt = v[j];
        }
        live = live && r.m != -INFINITY;
        float w[N];
        if (live) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float x = x_of(v[j], r.m, a.k);
                w[j] = exp2_fast(x);
                r.s += w[j];
                r.t = fmaf(w[j], fmaxf(x, kXMin), r.t);
            }
        }
        const bool good = live && fabsf(r.s) < INFINITY;             // no NaN, no +infinity
        const float none = live ? NAN : 0.f;
        if constexpr (kOp == kListTop) {
            logp_row(a, row, live, r, zt);
            int32_t* ids = a.top_ids + row * a.K;
            float* top = a.top_logp + row * a.K;
            int rank = 0, listed = 0;
            if (good) {
                rank = 1;
#pragma unroll
                for (int j = 0; j < N; ++j) rank += j < a.V && (v[j] > zt || (v[j] == zt && j < token));
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (!(v[j] > -INFINITY)) continue;
                    int place = 0;
#pragma unroll
                    for (int i = 0; i < N; ++i) place += v[i] > v[j] || (v[i] == v[j] && i < j);
                    ++listed;
                    if (place < a.K) {
                        ids[place] = j;
                        top[place] = log_prob(a, r, v[j]);
                    }
                }
            }
            for (int i = listed; i < a.K; ++i) {
                ids[i] = -1;
                top[i] = good ? -INFINITY : none;
            }
            if (a.rank) a.rank[row] = rank;
        } else {
            int at = -1;
            float mass = 0.f, t = 0.f;
            if (good && kOp == kListDrawAll) {
                // the first entry whose running mass exceeds u times the whole; the last one with a mass
                // where rounding leaves none
                const float target = u * r.s;
                float cum = 0.f;
                bool done = false;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    cum += w[j];
                    if (w[j] > 0.f && !done) {
                        at = j;
                        done = cum > target;
                    }
                }
                mass = r.s;
                t = r.t;
            }
            if (good && kOp == kListDraw) {
                // the mass before each entry of the first K; past them, none of theirs is kept
                float before[N], total = 0.f;
                int place[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    before[j] = 0.f;
                    place[j] = 0;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const bool first = v[i] > v[j] || (v[i] == v[j] && i < j);
                        place[j] += first;
                        before[j] += first ? w[i] : 0.f;
                    }
                    if (!(v[j] > -INFINITY)) place[j] = N;
                    if (place[j] < a.K) total += w[j];
                }
                int best = N + 1, last = -1;
                float target = 0.f;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (place[j] >= a.K || (place[j] > 0 && a.top_p < 1.f && !(before[j] < a.top_p * total))) place[j] = N;
                    if (place[j] < N) {
                        mass += w[j];
                        t = fmaf(w[j], fmaxf(x_of(v[j], r.m, a.k), kXMin), t);
                    }
                }
                target = u * mass;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (place[j] >= N || !(w[j] > 0.f)) continue;
                    if (before[j] + w[j] > target) {
                        if (place[j] < best) {
                            best = place[j];
                            at = j;
                        }
                    } else if (best > N && place[j] > last) {
                        at = j;
                    }
                    last = max(last, place[j]);
                }
            }
            float z_at = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j == at) z_at = v[j];
            if (good) write_draw(a, row, at, log_prob(a, r, z_at), row_entropy(r), log_prob(a, RowStat{r.m, mass, t}, z_at));
            else write_draw(a, row, -1, none, none, none);
        }
    }
}

template <class T, int kOp, int N>
cudaError_t launch_list_tiny(const ListArgs& a, int n_sm, cudaStream_t s) {
    const int64_t blocks = (a.n + kTinyThreads - 1) / kTinyThreads, most = 24 * (int64_t)n_sm;
    return launch_after(token_list_tiny_kernel<T, kOp, N>, (unsigned)(blocks < most ? blocks : most), kTinyThreads, 0, s, a);
}

}  // namespace

}  // namespace malib
