// Losses of token policies, short rows (up to 12 KB): a row is read once and its gradient
// written from where it is held. Up to 2 KB (8 KB for log-probabilities alone) that is the
// registers of G lanes of a warp, N vectors of 16 bytes each, beyond it a warp's part of
// shared memory. No barrier of the block: the lanes exchange maximum and sums by shuffles.
// Bound by instructions: some 15 an entry for both sweeps, and the row's loss, which takes
// more than the entries of the shortest rows: rows of up to 8 vectors take 8 lanes, so that
// a warp computes four rows' losses at once, and rows of a few entries one lane each.
// Measured on bf16 rows, policy loss with every term: 20,000 rows of 4,000 entries 69 us
// (280 MB: 4.1 TB/s), of 300 entries 20 us.
// The rows' shares of the statistics are summed by the lanes that take them, a fixed set
// of rows each, then by block and call in a fixed order.
#pragma once

#include "token_common.cuh"
#include "token_emit.cuh"
#include "token_top.cuh"

namespace malib {

namespace {

constexpr int kShortThreads = 128, kShortWarps = kShortThreads / 32;

template <int G>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The call's statistics from its threads' sums: by block, then in the block that ends last.
template <int kOp>
__device__ __forceinline__ void finish_short(const TokenArgs& a, Totals total) {
    total = block_totals<kShortThreads>(total);
    if (threadIdx.x == 0) a.part[blockIdx.x] = total;
    if (!last_of(a.ticket, gridDim.x)) return;
    const Totals v = sum_parts<kShortThreads>(a.part, (int)gridDim.x);
    if (threadIdx.x == 0) write_stats<kOp>(a, v);
}

// Blocks of `rows` rows at a time. Without statistics a few more than the SMs hold at once,
// which evens out the shares; with them, as many as they hold, because every block pays for
// the sum over its threads and for the count of those that have ended. Policy loss, us with
// 24 blocks an SM and with this: 20,000 bf16 rows of 300 entries 26.3 and 22.7, fp32 rows of
// 60 entries 20.6 and 16.5; without statistics 16.6 and 18.6.
template <class Kernel>
cudaError_t short_grid(Kernel kernel, size_t bytes, int64_t n, int64_t rows, bool stats, int n_sm, unsigned* out) {
    int64_t grid = (n + rows - 1) / rows, most = 24;
    if (stats && grid > 4 * (int64_t)n_sm) {
        int held = 0;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&held, kernel, kShortThreads, bytes);
        if (e != cudaSuccess) return e;
        most = held < 1 ? 1 : held;
    }
    if (grid > most * n_sm) grid = most * n_sm;
    if (grid > kTokenMaxCtas) grid = kTokenMaxCtas;
    *out = (unsigned)(grid < 1 ? 1 : grid);
    return cudaSuccess;
}

// From a row's statistics its results and its share of the call's, by the threads that hold
// them, `first` among them for what is stored; the gradient's factors c and whether it has any.
template <int kOp>
__device__ __forceinline__ void row_loss(const TokenArgs& a, int64_t row, bool first, const RowStat& r, float zt,
                                         const PpoRow& in, const Slopes& slopes, float w, const TopRow& top, bool& live,
                                         RowGrad& c, Totals& total) {
    if (kOp == kTokLogp) {
        if (first) logp_row(a, row, live, r, zt);
        return;
    }
    if (kOp == kTokScores || kOp == kTokScoresList) {
        if (live) c = scores_row(a, kOp == kTokScores ? slopes.g : top.q, slopes.e, r);
        if (kOp == kTokScores) c.at *= slopes.g;
        return;
    }
    RowSum sum{0.f, 0.f, 0.f, 0};
    float out = 0.f;
    if (kOp == kTokPpo) {
        if (live) {
            float loss, clipped, kl, H;
            out = log_prob(a, r, zt);
            c = ppo_row(a, in, r, out, w, &loss, &clipped, &kl, &H);
            sum = RowSum{w * loss, kl, H, clipped != 0.f ? 3 : 1};
        }
        if (first && a.logp) a.logp[row] = out;
    } else {
        live = live && top.live;
        if (live) {
            const float f = w * a.gscale * a.top_scale;
            out = top_loss(a, r, top);
            c = RowGrad{r.m, f / r.s, 0.f, f};
            sum = RowSum{w * out, out, 0.f, 1};
        }
        if (first && a.loss) a.loss[row] = out;
    }
    if (first) total.add(sum);
}

__device__ __forceinline__ void cp_async_16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

template <class T, int kOp, int G, int N>
__global__ void __launch_bounds__(kShortThreads) token_short_kernel(TokenArgs a) {
    constexpr int W = Elt<T>::W, kRows = 32 / G;     // rows a warp takes at a time
    constexpr bool kTop = has_list(kOp), kAll = kOp == kTokDistill;   // kAll: rows have no token
    static_assert(!kTop || G == 32, "a warp prepares its row's list");
    extern __shared__ TopEntry lists[];              // [warps][list_room]
    __shared__ uint32_t seen[kShortWarps][kTop ? 4096 / 32 : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % G;
    const int64_t step = (int64_t)gridDim.x * kShortWarps * kRows;
    Totals total{};
    wait_for_previous();
    if (kOp == kTokLogp) let_next_start();
    for (int64_t row0 = ((int64_t)blockIdx.x * kShortWarps + warp) * kRows; row0 < a.n; row0 += step) {
        const bool in_range = row0 + lane / G < a.n;
        const int64_t row = in_range ? row0 + lane / G : a.n - 1;
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        T* g = kOp != kTokLogp && a.g ? static_cast<T*>(a.g) + row * a.gld : nullptr;
        const int token = kAll ? -1 : a.tokens[row];
        const bool known = kAll || (token >= 0 && token < a.V);
        float w = 1.f;
        TokenRow pair{};
        PpoRow in{};
        if (has_stats(kOp)) w = a.weight ? a.weight[row] : a.w0;
        if (kOp == kTokPpo) in = ppo_load(a, row);
        if (kOp == kTokPairGrad) pair = a.rows[row];
        const bool read = in_range && w != 0.f && known && (kOp != kTokPairGrad || pair.inv_s != 0.f);
        if (!kAll && in_range && token >= a.V) atomicOr(a.err, ERRBIT_BAD_TOKEN);

        const int h = (int)(((uintptr_t)z & 15u) / sizeof(T));
        uint4 q[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int j = (sub + u * G) * W - h;
            q[u] = Elt<T>::none();
            if (!read || j >= a.V) continue;
            q[u] = j >= 0 && j + W <= a.V ? *reinterpret_cast<const uint4*>(z + j) : load_part(z, j, a.V);
        }
        float zt = 0.f;
        if (kOp != kTokPairGrad && !kAll && read) zt = Elt<T>::get(z[token]);
        const Slopes slopes = load_slopes<kOp>(a, row);
        TopEntry* list = lists + warp * list_room(kOp, a.top);
        TopRow top{};
        if constexpr (kTop) {
            if (read) top = list_row<T, kOp, 4096>(a, row, z, token, list, seen[warp]);
        }

        RowGrad c{0.f, 0.f, 0.f, 0.f};
        bool live = read;
        if (kOp == kTokPairGrad) {
            c = RowGrad{pair.m, -pair.value * pair.inv_s, 0.f, pair.value};
        } else {
            RowStat r{group_max<G>(vec_max<T>(q)), 0.f, 0.f};
            live = r.m != -INFINITY;
            if (live) gather<T>(r, q, a.k);
            r.s = group_sum<G>(r.s);
            r.t = group_sum<G>(r.t);
            row_loss<kOp>(a, row, sub == 0 && in_range, r, zt, in, slopes, w, top, live, c, total);
        }
        if (!g) continue;
        const bool alike = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0, plain = live && !(has_slope(kOp) && is_steep(c));
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int j = (sub + u * G) * W - h;
            if (!in_range || j >= a.V) continue;
            F2 v[W / 2] = {};
            if (plain) {
                emit<T, has_slope(kOp)>(q[u], c, a.k, v);
                if (!kTop && (unsigned)(token - j) < (unsigned)W) add_at(v, token - j, c.at);
            } else if (has_slope(kOp) && live) {
                emit_steep<T>(q[u], c, a.k, kTop ? -1 : token - j, v);
            }
            const uint4 out = Elt<T>::pack(v);
            if (alike && j >= 0 && j + W <= a.V) *reinterpret_cast<uint4*>(g + j) = out;
            else store_part(g + j, j, a.V, out);
        }
        if (kTop) {
            // the list's entries, over what the warp has written
            __syncwarp();
            if (live)
                for (int i = lane; i < list_room(kOp, a.top); i += 32) {
                    const TopEntry e = list[i];
                    if (e.id >= 0) g[e.id] = Elt<T>::put(list_entry<kOp>(e, c, a.k));
                }
            __syncwarp();
        }
    }
    if (has_stats(kOp) && a.stats) finish_short<kOp>(a, total);
}

// Rows of a warp each that pass through shared memory, more than 4 vectors a lane: every lane
// copies its vectors there and takes them from there in two short loops. Held in registers
// they need loops that are unrolled in full, with every vector's cases of a partial and of a
// shifted one: the instruction cache did not hold that (most stalls were for instructions),
// and 120 registers left 16 warps an SM. us, registers and this, policy loss of 20,000 bf16
// rows of 4,000 entries 92 and 71, of 3,001 97 and 64, of 1,500 with gradients aligned
// differently 69 and 45 (2,000: 41 and 44); of 1,001 (4 vectors a lane) 33 and 37. Without a
// gradient the loops are small: log-probabilities of 16,000 rows of 4,000 27 and 31.
template <class T, int kOp>
__global__ void __launch_bounds__(kShortThreads) token_slab_kernel(TokenArgs a, int slab) {
    constexpr int W = Elt<T>::W, kPer = 4;
    constexpr bool kTop = has_list(kOp), kAll = kOp == kTokDistill;   // kAll: rows have no token
    extern __shared__ __align__(16) uint8_t shared[];                // [warps][slab] vectors, [warps][list_room] entries
    __shared__ uint32_t seen[kShortWarps][kTop ? 4096 / 32 : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint4* own = reinterpret_cast<uint4*>(shared) + warp * slab;
    TopEntry* list = reinterpret_cast<TopEntry*>(shared + (size_t)kShortWarps * slab * 16) + warp * list_room(kOp, a.top);
    Totals total{};
    wait_for_previous();
    if (kOp == kTokLogp) let_next_start();
    for (int64_t row = (int64_t)blockIdx.x * kShortWarps + warp; row < a.n; row += (int64_t)gridDim.x * kShortWarps) {
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        T* g = kOp != kTokLogp && a.g ? static_cast<T*>(a.g) + row * a.gld : nullptr;
        const int token = kAll ? -1 : a.tokens[row];
        float w = 1.f;
        TokenRow pair{};
        PpoRow in{};
        if (has_stats(kOp)) w = a.weight ? a.weight[row] : a.w0;
        if (kOp == kTokPpo) in = ppo_load(a, row);
        if (kOp == kTokPairGrad) pair = a.rows[row];
        const bool known = kAll || (token >= 0 && token < a.V);
        const Slopes slopes = load_slopes<kOp>(a, row);
        bool live = w != 0.f && known && (kOp != kTokPairGrad || pair.inv_s != 0.f);
        if (!kAll && token >= a.V && lane == 0) atomicOr(a.err, ERRBIT_BAD_TOKEN);

        const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
        RowStat r{-INFINITY, 0.f, 0.f};
        float zt = 0.f;
        TopRow top{};
        if (live) {
            for (int i = lane; i < nv; i += 32) {
                const int j = i * W - h;
                if (j >= 0 && j + W <= a.V) cp_async_16(own + i, z + j);
                else own[i] = load_part(z, j, a.V);
            }
            if (kOp != kTokPairGrad && !kAll) zt = Elt<T>::get(z[token]);
            if constexpr (kTop) top = list_row<T, kOp, 4096>(a, row, z, token, list, seen[warp]);
            cp_async_wait();
            __syncwarp();
        }
        RowGrad c{0.f, 0.f, 0.f, 0.f};
        if (kOp == kTokPairGrad) {
            c = RowGrad{pair.m, -pair.value * pair.inv_s, 0.f, pair.value};
        } else {
            if (live) {
                for (int i0 = lane; i0 < nv; i0 += 32 * kPer) {
                    uint4 x[kPer];
#pragma unroll
                    for (int u = 0; u < kPer; ++u) x[u] = i0 + u * 32 < nv ? own[i0 + u * 32] : Elt<T>::none();
                    raise(r, vec_max<T>(x), a.k);
                    if (r.m != -INFINITY) gather<T>(r, x, a.k);
                }
                r = reduce_stat<32>(r, a.k);
                live = r.m != -INFINITY;
            }
            row_loss<kOp>(a, row, lane == 0, r, zt, in, slopes, w, top, live, c, total);
        }
        const bool plain = __all_sync(0xffffffffu, live && !(has_slope(kOp) && is_steep(c)));
        const int at = kTop ? -1 : token;            // a list has the token
        if (g && !plain) {
            if (has_slope(kOp) && live)
                emit_steep_part<T, 32>(lane, reinterpret_cast<const T*>(own) + h, 0, a.V, g, c, a.k, at);
            else
                zero_entries<T, 32>(lane, g, 0, a.V);
        }
        if (g && plain) {
            const uint8_t* src = reinterpret_cast<const uint8_t*>(own);
            const bool alike = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
            if (has_slope(kOp) && c.c1 != 0.f) emit_stage<T, true, 32, kPer>(lane, src, -h, 0, a.V, nv, g, alike, c, a.k, at);
            else emit_stage<T, false, 32, kPer>(lane, src, -h, 0, a.V, nv, g, alike, c, a.k, at);
        }
        if (kTop && g && live) {
            // the list's entries, over what the warp has written
            __syncwarp();
            for (int i = lane; i < list_room(kOp, a.top); i += 32) {
                const TopEntry e = list[i];
                if (e.id >= 0) g[e.id] = Elt<T>::put(list_entry<kOp>(e, c, a.k));
            }
        }
        __syncwarp();
    }
    if (has_stats(kOp) && a.stats) finish_short<kOp>(a, total);
}

// Rows of up to N <= 32 entries (the actions of the environments): a thread a row, so that
// its loss is computed once and not by every lane of a group. Rows that follow one another
// without a gap go through shared memory, so that neighbouring threads read and write
// neighbouring entries; others entry by entry. Bound by the launch and by instructions:
// 102,400 rows of 15 fp32 entries with every term of the policy loss took 26 us with 8
// lanes a row, 18 with a thread a row that reads its entries itself, and take 10 to 11 with this.
template <class T, int kOp, int N>
__global__ void __launch_bounds__(kShortThreads) token_tiny_kernel(TokenArgs a) {
    __shared__ T tile[kShortThreads * N];
    const int tid = threadIdx.x;
    const bool flat_z = a.ld == a.V, flat_g = a.gld == a.V;
    Totals total{};
    wait_for_previous();
    if (kOp == kTokLogp) let_next_start();
    for (int64_t row0 = (int64_t)blockIdx.x * kShortThreads; row0 < a.n; row0 += (int64_t)gridDim.x * kShortThreads) {
        const int rows = (int)min((int64_t)kShortThreads, a.n - row0), entries = rows * a.V;
        const bool in_range = tid < rows;
        const int64_t row = row0 + (in_range ? tid : 0);
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        T* g = kOp != kTokLogp && a.g ? static_cast<T*>(a.g) + row * a.gld : nullptr;
        if (flat_z) {
            const T* first = static_cast<const T*>(a.z) + row0 * a.V;
#pragma unroll 8
            for (int e = tid; e < entries; e += kShortThreads) tile[e] = first[e];
        }
        const int token = in_range ? a.tokens[row] : -1;
        float w = 1.f;
        TokenRow pair{};
        PpoRow in{};
        if (kOp == kTokPpo) {
            w = a.weight ? a.weight[row] : a.w0;
            in = ppo_load(a, row);
        }
        const Slopes slopes = load_slopes<kOp>(a, row);
        if (kOp == kTokPairGrad) pair = a.rows[row];
        const bool read = w != 0.f && token >= 0 && token < a.V && (kOp != kTokPairGrad || pair.inv_s != 0.f);
        if (token >= a.V) atomicOr(a.err, ERRBIT_BAD_TOKEN);
        float v[N];
        if (flat_z) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = read && j < a.V ? Elt<T>::get(tile[tid * a.V + j]) : -INFINITY;
            __syncthreads();
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = read && j < a.V ? Elt<T>::get(z[j]) : -INFINITY;
        }
        RowGrad c{0.f, 0.f, 0.f, 0.f};
        bool live = read;
        if (kOp == kTokPairGrad) {
            c = RowGrad{pair.m, -pair.value * pair.inv_s, 0.f, pair.value};
        } else {
            RowStat r{v[0], 0.f, 0.f};
            float zt = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                r.m = max_nan(r.m, v[j]);
                if (j == token) zt = v[j];
            }
            live = r.m != -INFINITY;
            if (live) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float x = x_of(v[j], r.m, a.k), e = exp2_fast(x);
                    r.s += e;
                    r.t = fmaf(e, fmaxf(x, kXMin), r.t);
                }
            }
            if (kOp == kTokLogp) {
                if (in_range) logp_row(a, row, live, r, zt);
            } else if (kOp == kTokScores) {
                if (live) c = scores_row(a, slopes.g, slopes.e, r);
                c.at *= slopes.g;
            } else {
                float logp = 0.f;
                if (live) {
                    float loss, clipped, kl, H;
                    logp = log_prob(a, r, zt);
                    c = ppo_row(a, in, r, logp, w, &loss, &clipped, &kl, &H);
                    total.add(RowSum{w * loss, kl, H, clipped != 0.f ? 3 : 1});
                }
                if (a.logp && in_range) a.logp[row] = logp;
            }
        }
        if (!g) continue;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (j >= a.V || !in_range) break;
            float f = 0.f;
            if (live) {
                if (is_steep(c)) {
                    f = emit_steep(v[j], c, a.k, j == token);
                } else {
                    const float x = x_of(v[j], c.m, a.k);
                    f = exp2_fast(x) * fmaf(c.c1, fmaxf(x, kXMin), c.c0);
                    if (j == token) f += c.at;
                }
            }
            if (flat_g) tile[tid * a.V + j] = Elt<T>::put(f);
            else g[j] = Elt<T>::put(f);
        }
        if (flat_g) {
            T* first = static_cast<T*>(a.g) + row0 * a.V;
            __syncthreads();
            for (int e = tid; e < entries; e += kShortThreads) first[e] = tile[e];
            __syncthreads();
        }
    }
    if (kOp == kTokPpo && a.stats) finish_short<kOp>(a, total);
}

template <class T, int kOp, int N>
cudaError_t launch_tiny(const TokenArgs& a, int n_sm, cudaStream_t s) {
    unsigned grid = 0;
    const cudaError_t e =
        short_grid(token_tiny_kernel<T, kOp, N>, 0, a.n, kShortThreads, kOp == kTokPpo && a.stats, n_sm, &grid);
    if (e != cudaSuccess) return e;
    return launch_after(token_tiny_kernel<T, kOp, N>, grid, kShortThreads, 0, s, a);
}

template <class T, int kOp, int G, int N>
cudaError_t launch_short(const TokenArgs& a, int n_sm, cudaStream_t s) {
    const size_t bytes = has_list(kOp) ? (size_t)kShortWarps * list_room(kOp, a.top) * sizeof(TopEntry) : 0;
    if (bytes > 0) {
        const cudaError_t e = cudaFuncSetAttribute(token_short_kernel<T, kOp, G, N>,
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   kShortWarps * list_room(kOp, kTokenMaxTop) * (int)sizeof(TopEntry));
        if (e != cudaSuccess) return e;
    }
    unsigned grid = 0;
    const bool stats = has_stats(kOp) && a.stats;
    const cudaError_t e =
        short_grid(token_short_kernel<T, kOp, G, N>, bytes, a.n, kShortWarps * (32 / G), stats, n_sm, &grid);
    if (e != cudaSuccess) return e;
    return launch_after(token_short_kernel<T, kOp, G, N>, grid, kShortThreads, bytes, s, a);
}

template <class T, int kOp>
cudaError_t launch_slab(const TokenArgs& a, int nv, int n_sm, cudaStream_t s) {
    const int slab = (nv + 31) / 32 * 32;
    const size_t bytes = (size_t)kShortWarps * (slab * 16 + list_room(kOp, a.top) * sizeof(TopEntry));
    cudaError_t e = cudaFuncSetAttribute(token_slab_kernel<T, kOp>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         kShortWarps * (kShortVecs * 16 + list_room(kOp, kTokenMaxTop) * (int)sizeof(TopEntry)));
    if (e != cudaSuccess) return e;
    unsigned grid = 0;
    const bool stats = has_stats(kOp) && a.stats;
    e = short_grid(token_slab_kernel<T, kOp>, bytes, a.n, kShortWarps, stats, n_sm, &grid);
    if (e != cudaSuccess) return e;
    return launch_after(token_slab_kernel<T, kOp>, grid, kShortThreads, bytes, s, a, slab);
}

// Lanes a row and vectors a lane by the most vectors a row has.
template <class T, int kOp>
cudaError_t launch_short_op(const TokenArgs& a, int n_sm, cudaStream_t s) {
    const int nv = (a.V + 2 * Elt<T>::W - 2) / Elt<T>::W;
    if constexpr (!has_list(kOp)) {
        if (a.V <= 8) return launch_tiny<T, kOp, 8>(a, n_sm, s);
        if (a.V <= 16) return launch_tiny<T, kOp, 16>(a, n_sm, s);
        if (a.V <= 32) return launch_tiny<T, kOp, 32>(a, n_sm, s);
        if (nv <= 8) return launch_short<T, kOp, 8, 1>(a, n_sm, s);
    }
    if (nv <= 32) return launch_short<T, kOp, 32, 1>(a, n_sm, s);
    if (nv <= 64) return launch_short<T, kOp, 32, 2>(a, n_sm, s);
    if (nv <= 128) return launch_short<T, kOp, 32, 4>(a, n_sm, s);
    if constexpr (kOp == kTokLogp) {
        if (nv <= 256) return launch_short<T, kOp, 32, 8>(a, n_sm, s);
        if (nv <= 512) return launch_short<T, kOp, 32, 16>(a, n_sm, s);
    }
    return launch_slab<T, kOp>(a, nv, n_sm, s);
}

template <class T>
cudaError_t launch_short_type(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    if (op == kTokLogp) return launch_short_op<T, kTokLogp>(a, n_sm, s);
    if (op == kTokPpo) return launch_short_op<T, kTokPpo>(a, n_sm, s);
    if (op == kTokDistill) return launch_short_op<T, kTokDistill>(a, n_sm, s);
    if (op == kTokScores) return launch_short_op<T, kTokScores>(a, n_sm, s);
    if (op == kTokScoresList) return launch_short_op<T, kTokScoresList>(a, n_sm, s);
    return launch_short_op<T, kTokPairGrad>(a, n_sm, s);
}

}  // namespace

}  // namespace malib
