// Draws from the whole of many rows, as a stream. A warp of a CTA (the producer) claims rows and copies them in
// batches into a ring of stages; four (the sweepers) gather a row's statistics and the sums of its
// segments; and one more (the finisher) finds the row's token from those, while the sweepers are at the next
// row. A row has two places to pass through, and no warp waits for another but through the ring and
// these. 16,384 rows of 32,768 bf16 entries 168 us (6.4 TB/s), by a block of 128 threads a row 218; 8,192 of
// 65,536, a quarter left out, 125 and 137. Rows that start inside a vector cost two loads from shared memory a
// vector: 8,192 rows of 50,256 entries 128 us, of 50,257 138 (129 when sums took the memory's vectors); the
// second by a shuffle from the next lane 147. (Lists were no faster this way, with one to four finishers: a row's
// selection has half as many instructions as its sums.)
//
// Every wait is bounded; one that expires ends the CTA's work and is reported as MALIB_ETIMEOUT.
#pragma once

#include "token_list.cuh"

namespace malib {

namespace {

constexpr int kSweepers = 4, kSweepThreads = 32 * kSweepers, kStreamThreads = kSweepThreads + 64;
constexpr int kStreamBatch = kSweepThreads * kListPer;               // vectors of a stage: a segment for each sweeper
constexpr int kStageBytes = (kStreamBatch + 1) * 16;                 // one more where the row starts inside a vector
constexpr int kStreamStages = 2, kStreamCtas = 4, kPlaces = 2;       // of a CTA; CTAs an SM
constexpr int kStreamMostBatches = 1024;             // of a row: 4 segments of 8 bytes each, in two places

// The ring's present stage, and the parity of its use.
struct Stage {
    int at = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() {
        if (++at == kStreamStages) {
            at = 0;
            parity ^= 1u;
        }
    }
};
// A place for a row, from the sweepers to the finisher.
struct __align__(16) StreamPlace {
    RowStat stat[kSweepers];
    float u;                                         // the row's random number
    int64_t row;                                     // < 0: no more
};

template <class T, class Own>
__global__ void __launch_bounds__(kStreamThreads, kStreamCtas) token_draw_stream_kernel(ListArgs a, int batches) {
    constexpr int W = Elt<T>::W, kWarpVecs = kSegmentVecs;
    extern __shared__ __align__(128) uint8_t dynamic[];              // stages, then by place the segments' (m, S)
    __shared__ __align__(8) uint64_t full[kStreamStages], empty[kStreamStages], swept[kPlaces], freed[kPlaces];
    __shared__ int64_t stage_row[kStreamStages];     // < 0: no more
    __shared__ StreamPlace place[kPlaces];
    __shared__ int dead;                             // a bounded wait has expired: nothing waits any more
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float2* segment = reinterpret_cast<float2*>(dynamic + kStreamStages * kStageBytes);
    if (tid == 0) {
        dead = 0;
        for (int i = 0; i < kStreamStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], kSweepers);
        }
        for (int i = 0; i < kPlaces; ++i) {
            mbar_init(&swept[i], kSweepers);
            mbar_init(&freed[i], 1);
        }
        fence_proxy_async_smem();
    }
    __syncthreads();
    wait_for_previous();
    let_next_start();
    volatile int* gone = &dead;
    const auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (mbar_try_wait(bar, parity) || *gone) return;
        if (!mbar_wait_bounded(bar, parity, kWaitLimitNs)) {
            *gone = 1;
            atomicOr(a.err, ERRBIT_TIMEOUT);
        }
    };

    if (warp == kSweepers) {
        // ---- producer: the next row is claimed, and its token asked for, a row ahead
        const auto claim = [&] { return lane == 0 ? (int64_t)gridDim.x + (int64_t)atomicAdd(a.claims, 1ull) : 0ll; };
        const auto token_of = [&](int64_t row) { return row < a.n && a.tokens ? a.tokens[row] : 0; };
        int64_t row = blockIdx.x, next = __shfl_sync(0xffffffffu, claim(), 0);
        int token = token_of(row);
        Stage at, issued;
        bool any = false, wrapped = false;
        while (row < a.n && !*gone) {
            const int64_t after = claim();
            const int next_token = token_of(next);
            if (token < 0) {
                if (lane == 0) write_draw(a, row, -1, 0.f, 0.f, 0.f);
            } else {
                const T* z = static_cast<const T*>(a.z) + row * a.ld;
                const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
                // nv: the memory's vectors, of which a row that starts inside one has one more than its own may need
                for (int v = 0; v * W < a.V; v += kStreamBatch) {
                    const int n = min(kStreamBatch + (h > 0 ? 1 : 0), nv - v);
                    uint8_t* dst = dynamic + at.at * kStageBytes;
                    // a partial first (lanes 0 ..) or last (lanes 16 ..) vector of the row
                    const bool head = v == 0 && h > 0, tail = v + n == nv && (h + a.V) % W != 0;
                    const int pv = lane < 16 ? 0 : nv - 1, pj = pv * W - h + (lane & 15);
                    const bool fill = (lane & 15) < W && (lane < 16 ? head : tail);
                    T entry = Elt<T>::put(-INFINITY);
                    if (fill && pj >= 0 && pj < a.V) entry = z[pj];
                    wait(&empty[at.at], at.parity ^ 1u);
                    if (fill) reinterpret_cast<T*>(dst)[(pv - v) * W + (lane & 15)] = entry;
                    // behind the row's last one, which the row's own last one is put together with
                    const bool behind = lane == 15 && h > 0 && n <= kStreamBatch;
                    if (behind) *reinterpret_cast<uint4*>(dst + n * 16) = Elt<T>::none();
                    if (fill || behind) fence_proxy_async_smem();    // a later use's copy overwrites what is stored here
                    __syncwarp();
                    if (*gone) break;
                    any = true;
                    wrapped |= at.at + 1 == kStreamStages;
                    issued = at;
                    if (lane == 0) {
                        stage_row[at.at] = row;
                        const int b0 = head ? 1 : 0, b1 = tail ? n - 1 : n;
                        const uint32_t bytes = b1 > b0 ? (uint32_t)(b1 - b0) * 16u : 0u;
                        mbar_arrive_expect_tx(&full[at.at], bytes);
                        if (bytes) bulk_g2s(dst + b0 * 16, z + ((int64_t)(v + b0) * W - h), bytes, &full[at.at]);
                    }
                    __syncwarp();
                    at.next();
                }
            }
            row = next;
            token = next_token;
            next = __shfl_sync(0xffffffffu, after, 0);
        }
        wait(&empty[at.at], at.parity ^ 1u);
        if (!*gone && lane == 0) {
            stage_row[at.at] = -1;
            mbar_arrive_release(&full[at.at]);
        }
        __syncwarp();
        if (*gone && any)                            // copies in flight end before the block does
            for (int i = 0; i < kStreamStages; ++i)
                if (wrapped || i <= issued.at)
                    mbar_wait_bounded(&full[i], i <= issued.at ? issued.parity : issued.parity ^ 1u, 1000000);
    } else if (warp < kSweepers) {
        // ---- sweepers
        const float low_reach = 160.f / a.k;
        Stage at;
        for (uint32_t turn = 0;; ++turn) {
            const int f = turn % kPlaces;
            wait(&full[at.at], at.parity);
            if (*gone) break;
            const int64_t row = stage_row[at.at];
            wait(&freed[f], (turn / kPlaces & 1u) ^ 1u);             // (the parity of the place's use)
            if (row < 0) {
                __syncwarp();
                if (lane == 0) {
                    if (warp == 0) place[f].row = -1;
                    mbar_arrive_release(&swept[f]);
                }
                break;
            }
            const T* z = static_cast<const T*>(a.z) + row * a.ld;
            const int by = (int)((uintptr_t)z & 15u), nv = (a.V + W - 1) / W;        // vectors by their entries' index
            const uint32_t bits = 8u * (by & 3);
            RowUniform random{};
            if (warp == 0) random = load_uniform(a, row);
            Own st{};
            st.m = -INFINITY;
            float2* sums = segment + f * batches * kSweepers + warp;
            for (int b = 0; b < nv; b += kStreamBatch, sums += kSweepers) {
                if (b > 0) wait(&full[at.at], at.parity);
                const uint4* in = reinterpret_cast<const uint4*>(dynamic + at.at * kStageBytes) + warp * kWarpVecs + lane;
                const int from = b + warp * kWarpVecs + lane;        // the thread's first
                uint4 x[kListPer];
                if (by == 0) {
#pragma unroll
                    for (int u = 0; u < kListPer; ++u) x[u] = in[u * 32];
                } else {
                    by_word(by, [&](auto word) {
#pragma unroll
                        for (int u = 0; u < kListPer; ++u) x[u] = shifted<decltype(word)::at>(in[u * 32], in[u * 32 + 1], bits);
                    });
                }
                if (b + (warp + 1) * kWarpVecs > nv) {               // what the stage has behind the row
#pragma unroll
                    for (int u = 0; u < kListPer; ++u)
                        if (from + u * 32 >= nv) x[u] = Elt<T>::none();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_release(&empty[at.at]);
                at.next();
                const float mx = warp_max(vec_max<T>(x));
                const float s = sum_segment<T>(st, x, mx, a.k, low_reach);
                if (lane == 0) *sums = make_float2(mx, s);
            }
            RowStat r = stat_of(st);
            r.s = warp_add(r.s);
            r.t = warp_add(r.t);
            if (lane == 0) {
                place[f].stat[warp] = r;
                if (warp == 0) {
                    place[f].row = row;
                    place[f].u = uniform_of(a, random);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_release(&swept[f]);
        }
    } else {
        // ---- finisher
        for (uint32_t turn = 0;; ++turn) {
            const int f = turn % kPlaces;
            wait(&swept[f], turn / kPlaces & 1u);
            if (*gone) break;
            const int64_t row = place[f].row;
            if (row < 0) break;
            const T* z = static_cast<const T*>(a.z) + row * a.ld;
            const RowStat r = reduce_stat<kSweepers>(place[f].stat[lane & (kSweepers - 1)], a.k);
            const bool live = r.m != -INFINITY;
            if (live && fabsf(r.s) < INFINITY) {     // no NaN, no +infinity
                draw_all<T>(a, row, r, IndexView<T>{z, a.V}, segment + f * batches * kSweepers, place[f].u,
                            [](int) { return true; }, lane);
            } else if (lane == 0) {
                write_draw(a, row, -1, live ? NAN : 0.f, live ? NAN : 0.f, live ? NAN : 0.f);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_release(&freed[f]);
        }
    }
    // the CTA that ends last clears the claims for the next call
    if (last_of(a.ticket, gridDim.x) && tid == 0) *a.claims = 0ull;
}

template <class T, class Own>
cudaError_t launch_draw_stream_as(const ListArgs& a, int batches, int n_sm, cudaStream_t s) {
    const auto kernel = token_draw_stream_kernel<T, Own>;
    const size_t bytes = (size_t)kStreamStages * kStageBytes + (size_t)kPlaces * batches * kSweepers * sizeof(float2);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kListMost);
    if (e != cudaSuccess) return e;
    int held = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&held, kernel, kStreamThreads, bytes);
    if (e != cudaSuccess) return e;
    const int64_t most = (int64_t)(held < 1 ? 1 : held) * n_sm;
    return launch_after(kernel, (unsigned)(a.n < most ? a.n : most), kStreamThreads, bytes, s, a, batches);
}
template <class T>
cudaError_t launch_draw_stream(const ListArgs& a, int64_t nv, int n_sm, cudaStream_t s) {
    const int batches = (int)((nv + kStreamBatch - 1) / kStreamBatch);
    return batches > kManyBatches ? launch_draw_stream_as<T, LongStat>(a, batches, n_sm, s)
                                  : launch_draw_stream_as<T, RowStat>(a, batches, n_sm, s);
}

}  // namespace

}  // namespace malib
