// Lists and draws of rows of up to 4 KB: a warp a row, its entries in registers.
// Lists sort the entries from a bound on, which has at least K from it on and few more: bisected among the
// values between the smallest of the lanes' maxima, from which on there are 32 entries at least, and the
// row's maximum.
// Bound by instructions (8,192 rows of 2,000 bf16 entries, lists of 64: issue slots 54 %, 27 us, of 250 109 us, by
// exchanges in 16 registers): a warp needs no barrier, and no entry is read twice. Blocks of a warp, which went
// by the longer rows' way, took 53 and 650 us; 102,400 draws from 100 fp32 entries 108, now 42.
#pragma once

#include "token_list.cuh"

namespace malib {

namespace {

constexpr int kRowWarps = 4;                         // rows of a CTA
constexpr int kShortTop = 128;                       // entries of lists that are sorted in 8 registers or fewer

// Larger for larger entries of a type, the same for -0 and 0; the entry of a key; the key of the lowest finite one.
// With the index they are sorted as Sorted, largest first.
template <class T>
struct ShortKey;
template <>
struct ShortKey<float> {
    using Sorted = uint64_t;
    static constexpr uint32_t kLowest = 0x00800000u;
    __device__ static uint32_t of(float z) { return order_key(z); }
    __device__ static float value(uint32_t key) { return order_value(key); }
    __device__ static Sorted sorted(float z, int j) { return (uint64_t)of(z) << 32 | (0xffffffffu - (uint32_t)j); }
    __device__ static uint64_t entry(Sorted k) { return k >> 32 << 24 | (k & kIndexMask); }
};
template <class T>
struct HalfKey {
    using Sorted = uint32_t;
    __device__ static Sorted sorted(float z, int j) { return ShortKey<T>::of(z) << 16 | (0xffffu - (uint32_t)j); }
    __device__ static uint64_t entry(Sorted k) { return entry_key(ShortKey<T>::value(k >> 16), 0xffff - (int)(k & 0xffffu)); }
};
template <>
struct ShortKey<__nv_bfloat16> : HalfKey<__nv_bfloat16> {
    static constexpr uint32_t kLowest = 0x0080u;
    __device__ static uint32_t of(float z) { return order_key(z) >> 16; }
    __device__ static float value(uint32_t key) {
        return __uint_as_float((key & 0x8000u ? key ^ 0x8000u : ~key & 0xffffu) << 16);
    }
};
template <>
struct ShortKey<__half> : HalfKey<__half> {
    static constexpr uint32_t kLowest = 0x0400u;
    __device__ static uint32_t of(float z) {
        const uint32_t b = __half_as_ushort(__float2half_rn(__fadd_rn(z, 0.f)));
        return b & 0x8000u ? ~b & 0xffffu : b | 0x8000u;
    }
    __device__ static float value(uint32_t key) {
        return __half2float(__ushort_as_half((unsigned short)(key & 0x8000u ? key ^ 0x8000u : ~key)));
    }
};

// kLong: lists of more than kShortTop entries.
template <int kOp, bool kLong>
struct ShortRow {
    static constexpr int kCap = kLong ? kTokenMaxTop : 2 * kShortTop;                // keys that are sorted
    uint16_t index[kCap];
    uint64_t list[kOp != kListDraw ? 1 : kLong ? kTokenMaxTop : kShortTop];
};

template <class T, int N>
__device__ __forceinline__ uint32_t count_from(const uint4 (&x)[N], float z) {
    Above<T> above;
    const uint32_t thr = Above<T>::both(z);
#pragma unroll
    for (int u = 0; u < N; ++u) above.add(x[u], thr);
    return __reduce_add_sync(0xffffffffu, above.take());
}
__device__ __forceinline__ float warp_min(float v) {
    float r;
    asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// Bits of a lane's entries that are >= a threshold. 32-bit types: of entry i of vector u bit 4 u + i of a; 16-bit
// types: of the even and odd entries of word w = 4 u + i bits w and w + 16 of a, for w >= 16 of b.
struct Hits {
    uint32_t a = 0, b = 0;
};
template <class T, int N>
__device__ __forceinline__ Hits hits_from(const uint4 (&x)[N], float z) {
    Hits r;
    const uint32_t thr = Above<T>::both(z);
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 4 * u + i;
            if constexpr (sizeof(T) == 4) r.a |= Above<float>::mask(w[i], thr) & 1u << at;
            else if (at < 16) r.a |= Above<T>::mask(w[i], thr) & 0x10001u << at;
            else r.b |= Above<T>::mask(w[i], thr) & 0x10001u << (at - 16);
        }
    }
    return r;
}
// The entry of a bit, as if lane 0's.
template <class T>
__device__ __forceinline__ int hit_index(int bit, int more) {
    if (sizeof(T) == 4) return (bit >> 2) * 128 + (bit & 3);
    const int w = (bit & 15) + more;
    return (w >> 2) * 256 + 2 * (w & 3) + (bit >> 4);
}
template <class T, class Row>
__device__ __forceinline__ uint32_t push_hits(Row& s, Hits hits, uint32_t base, int first, int lane) {
    const uint32_t own = __popc(hits.a) + __popc(hits.b);
    uint32_t upto = own;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t q = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += q;
    }
    uint32_t to = base + upto - own;
    for (; hits.a; hits.a &= hits.a - 1, ++to)
        if (to < (uint32_t)Row::kCap) s.index[to] = (uint16_t)(first + hit_index<T>(__ffs(hits.a) - 1, 0));
    for (; hits.b; hits.b &= hits.b - 1, ++to)
        if (to < (uint32_t)Row::kCap) s.index[to] = (uint16_t)(first + hit_index<T>(__ffs(hits.b) - 1, 16));
    return base + __shfl_sync(0xffffffffu, upto, 31);
}

// Sorts 32 R keys of a warp, largest first; key i is in register i / 32 of lane i % 32.
template <int R, class K>
__device__ __forceinline__ void sort_warp(K (&key)[R], int lane) {
#pragma unroll(R <= 4 ? 7 : 1)
    for (int size = 2; size <= 32 * R; size *= 2) {
#pragma unroll
        for (int gap = 16 * R; gap >= 32; gap /= 2) {
            if (gap >= size) continue;
#pragma unroll
            for (int q = 0; q < R; ++q) {
                if ((q & gap / 32) != 0) continue;
                const K x = key[q], y = key[q + gap / 32];
                const bool falls = (32 * q & size) == 0;
                key[q] = falls ? max(x, y) : min(x, y);
                key[q + gap / 32] = falls ? min(x, y) : max(x, y);
            }
        }
#pragma unroll(R <= 4 ? 5 : 1)
        for (int gap = min(16, size / 2); gap > 0; gap /= 2) {
#pragma unroll
            for (int q = 0; q < R; ++q) {
                const K other = __shfl_xor_sync(0xffffffffu, key[q], gap);
                const bool falls = ((32 * q + lane) & size) == 0, first = (lane & gap) == 0;
                key[q] = falls == first ? max(key[q], other) : min(key[q], other);
            }
        }
    }
}

// f(place, key) for the first K of the n entries whose indexes are in s.index.
template <class T, int R, class Row, class F>
__device__ __forceinline__ void each_listed(const Row& s, const T* z, int n, int K, int lane, F f) {
    using Key = ShortKey<T>;
    typename Key::Sorted key[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
        const int i = 32 * q + lane, j = i < n ? s.index[i] : 0;
        key[q] = i < n ? Key::sorted(Elt<T>::get(z[j]), j) : 0;
    }
    sort_warp<R>(key, lane);
#pragma unroll
    for (int q = 0; q < R; ++q)
        if (32 * q + lane < min(n, K)) f(32 * q + lane, Key::entry(key[q]));
}

// The first K entries of a row z (a warp's): f(place, key) of each; how many there are. Its entries have no NaN
// and no +infinity, and m, the largest, is finite. x: a lane's vectors, vmax: the largest of each.
template <class T, int N, class Row, class F>
__device__ __forceinline__ int list_row(Row& s, const T* z, const uint4 (&x)[N], const float (&vmax)[N], float m, int h, int K,
                                        int lane, F f) {
    using Key = ShortKey<T>;
    constexpr int W = Elt<T>::W;
    // a bound with K entries from it on (or the lowest value), and how many there are: 32 are from the lanes'
    // maxima on, 64 from their second vectors'
    float most = vmax[0], second = -INFINITY;
#pragma unroll
    for (int u = 1; u < N; ++u) {
        second = fmaxf(second, fminf(most, vmax[u]));
        most = fmaxf(most, vmax[u]);
    }
    uint32_t lo = Key::kLowest, hi = Key::of(m) + 1;
    const float from = warp_min(K <= 32 ? most : second);
    if (K <= 64 && from > -INFINITY) lo = Key::of(from);
    uint32_t n = count_from<T>(x, Key::value(lo));
    // what is sorted in 1, 2, 4, .. registers
    const uint32_t enough = K <= 24 ? 32 : K <= 52 ? 64 : K <= 104 ? 128 : K <= 232 ? 256 : K <= 480 ? 512 : Row::kCap;
    while (n > enough && hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2, c = count_from<T>(x, Key::value(mid));
        if (c >= (uint32_t)K) {
            lo = mid;
            n = c;
        } else {
            hi = mid;
        }
    }
    const int first = lane * W - h;
    if (n <= (uint32_t)Row::kCap) {
        push_hits<T>(s, hits_from<T>(x, Key::value(lo)), 0, first, lane);
    } else {
        // many equal ones at the bound (hi is lo's next, and fewer than K are from it on): the first of them
        uint32_t base = hi > Key::of(m) ? 0u : push_hits<T>(s, hits_from<T>(x, Key::value(hi)), 0, first, lane);
        const float bound = Key::value(lo);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            uint32_t equal = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) equal |= entry_of<T>(x[u], i) == bound ? 1u << i : 0u;
            uint32_t upto = __popc(equal);
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t q = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += q;
            }
            uint32_t to = base + upto - __popc(equal);
            for (; equal; equal &= equal - 1, ++to)
                if (to < (uint32_t)Row::kCap) s.index[to] = (uint16_t)(first + u * 32 * W + __ffs(equal) - 1);
            base += __shfl_sync(0xffffffffu, upto, 31);
        }
        n = Row::kCap;
    }
    __syncwarp();
    if constexpr (Row::kCap <= 256) {
        if (n <= 32) each_listed<T, 1>(s, z, (int)n, K, lane, f);
        else if (n <= 64) each_listed<T, 2>(s, z, (int)n, K, lane, f);
        else if (n <= 128) each_listed<T, 4>(s, z, (int)n, K, lane, f);
        else each_listed<T, 8>(s, z, (int)n, K, lane, f);
    } else {
        if (n <= 256) each_listed<T, 8>(s, z, (int)n, K, lane, f);
        else if (n <= 512) each_listed<T, 16>(s, z, (int)n, K, lane, f);
        else each_listed<T, 32>(s, z, (int)n, K, lane, f);
    }
    __syncwarp();
    return min((int)n, K);
}

// CTAs an SM: as many as registers last for.
template <class T, int kOp, int N, bool kLong>
constexpr int short_ctas() {
    if (kLong) return sizeof(T) == 4 ? 3 : 4;
    return sizeof(T) == 4 && kOp != kListDrawAll ? (N == 1 ? 9 : N == 2 ? 8 : N == 4 ? 6 : 4) : N <= 2 ? 12 : N == 4 ? 9 : 7;
}

template <class T, int kOp, int N, bool kLong>
__global__ void __launch_bounds__(32 * kRowWarps, short_ctas<T, kOp, N, kLong>()) token_list_short_kernel(ListArgs a) {
    constexpr int W = Elt<T>::W;
    using Row = ShortRow<kOp, kLong>;
    __shared__ Row shared[kOp == kListDrawAll ? 1 : kRowWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Row& s = shared[kOp == kListDrawAll ? 0 : warp];
    wait_for_previous();
    let_next_start();
    const int64_t step = (int64_t)gridDim.x * kRowWarps;
    int64_t row = (int64_t)blockIdx.x * kRowWarps + warp;
    int token = row < a.n && a.tokens ? a.tokens[row] : 0;
    for (; row < a.n; row += step) {
        const int next_token = row + step < a.n && a.tokens ? a.tokens[row + step] : 0;
        const int own_token = token;
        token = next_token;
        bool live = own_token >= 0;
        if (kOp == kListTop && own_token >= a.V) {
            live = false;
            if (lane == 0) atomicOr(a.err, ERRBIT_BAD_TOKEN);
        }
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
        // the row's whole vectors; a partial first or last one is filled up
        const int full_lo = h > 0 ? 1 : 0, full_hi = (h + a.V) % W != 0 ? nv - 1 : nv;
        const uint32_t full = (uint32_t)max(0, full_hi - full_lo);
        const uint4* src = reinterpret_cast<const uint4*>(z - h);
        uint4 x[N];
        float vmax[N], zt = 0.f, u01 = 0.f;
        RowStat r{-INFINITY, 0.f, 0.f};
        if (live) {
            if (kOp == kListTop && a.tokens) zt = Elt<T>::get(z[own_token]);
            if (kOp == kListDrawAll) u01 = row_uniform(a, row);
#pragma unroll
            for (int u = 0; u < N; ++u)
                x[u] = (uint32_t)(u * 32 + lane - full_lo) < full ? src[u * 32 + lane] : Elt<T>::none();
            const int tail = full_hi < nv ? nv - 1 : -1;
            if (lane == 0 && full_lo > 0) x[0] = load_part(z, -h, a.V);
            if (tail >= full_lo && lane == tail % 32) {
                const uint4 q = load_part(z, tail * W - h, a.V);
#pragma unroll
                for (int u = 0; u < N; ++u)
                    if (u == tail / 32) x[u] = q;
            }
            // (draws from the whole row: the same sums wherever it lies)
            if (kOp == kListDrawAll && h > 0) realign<T>(x, Elt<T>::none(), (int)((uintptr_t)z & 15u), lane);
#pragma unroll
            for (int u = 0; u < N; ++u) {
                vmax[u] = Elt<T>::largest(Elt<T>::max(Elt<T>::max(x[u].x, x[u].y), Elt<T>::max(x[u].z, x[u].w)));
                r.m = max_nan(r.m, vmax[u]);
            }
            r.m = warp_max(r.m);
            live = r.m != -INFINITY;
        }
        float sum[N];                                // of a vector
        if (live) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                RowStat part{r.m, 0.f, 0.f};
                gather<T>(part, reinterpret_cast<const uint4(&)[1]>(x[u]), a.k);
                sum[u] = part.s;
                r.s += part.s;
                r.t += part.t;
            }
            r.s = warp_add(r.s);
            r.t = warp_add(r.t);
        }
        const bool good = live && fabsf(r.s) < INFINITY;             // no NaN, no +infinity
        const float none = live ? NAN : 0.f;
        if constexpr (kOp == kListTop) {
            if (a.rank) {
                // entries that come before the token's
                uint32_t before = 0;
                if (good) {
                    const uint32_t thr_before = Above<T>::both(zt), thr_behind = Above<T>::both(Above<T>::next(zt));
                    Above<T> above;
#pragma unroll
                    for (int u = 0; u < N; ++u) {
                        const int j = (u * 32 + lane) * W - h;
                        if (zt == -INFINITY) {       // after every unmasked entry, and the masked ones before it
#pragma unroll
                            for (int i = 0; i < W; ++i)
                                before += j + i >= 0 && j + i < a.V && (entry_of<T>(x[u], i) > -INFINITY || j + i < own_token);
                        } else {
                            above.add(x[u], j + W <= own_token ? thr_before : thr_behind);
                            if (j < own_token && j + W > own_token)
#pragma unroll
                                for (int i = 0; i < W; ++i) before += j + i < own_token && entry_of<T>(x[u], i) == zt;
                        }
                    }
                    before += above.take();
                    before = __reduce_add_sync(0xffffffffu, before);
                }
                if (lane == 0) a.rank[row] = good ? (int)before + 1 : 0;
            }
            if (lane == 0) logp_row(a, row, live, r, zt);
        }
        if (!good) {
            if (kOp == kListTop) {
                for (int i = lane; i < a.K; i += 32) {
                    a.top_ids[row * a.K + i] = -1;
                    a.top_logp[row * a.K + i] = none;
                }
            } else if (lane == 0) {
                write_draw(a, row, -1, none, none, none);
            }
            continue;
        }
        if constexpr (kOp == kListDrawAll) {
            // the vector whose running mass passes the target, the last one with a mass where rounding leaves none
            const float target = u01 * r.s;
            float passed = 0.f, before = 0.f;
            int at = -1, at_lane = 0;
            bool hit = false;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const float cum = warp_scan(sum[u], lane);
                const unsigned over = __ballot_sync(0xffffffffu, sum[u] > 0.f && passed + cum > target),
                               some = __ballot_sync(0xffffffffu, sum[u] > 0.f);
                if (!hit && some) {
                    hit = over != 0;
                    at = u;
                    at_lane = hit ? __ffs(over) - 1 : 31 - __clz(some);
                    before = passed + (cum - sum[u]);                // (of lane at_lane)
                }
                passed += __shfl_sync(0xffffffffu, cum, 31);
            }
            if (lane == at_lane) {
                float found = -INFINITY;
                int j = -1;
                bool done = false;
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    if (u != at) continue;
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float e = entry_of<T>(x[u], i), w = exp2_fast(x_of(e, r.m, a.k));
                        before += w;
                        if (w > 0.f && !done) {
                            found = e;
                            j = (u * 32 + lane) * W + i;
                            done = before > target;
                        }
                    }
                }
                const float logp = log_prob(a, r, found);
                write_draw(a, row, j, logp, row_entropy(r), logp);
            }
        } else {
            if constexpr (kOp == kListDraw) {
                const int n = list_row<T, N>(s, z, x, vmax, r.m, h, a.K, lane, [&](int i, uint64_t key) { s.list[i] = key; });
                draw_listed(a, row, r, s.list, n, lane);
            } else {
                const int n = list_row<T, N>(s, z, x, vmax, r.m, h, a.K, lane, [&](int i, uint64_t key) {
                    a.top_ids[row * a.K + i] = key_index(key);
                    a.top_logp[row * a.K + i] = log_prob(a, r, key_logit(key));
                });
                for (int i = n + lane; i < a.K; i += 32) {
                    a.top_ids[row * a.K + i] = -1;
                    a.top_logp[row * a.K + i] = -INFINITY;
                }
            }
            __syncwarp();
        }
    }
}

template <class T, int kOp, int N, bool kLong>
cudaError_t launch_list_short_as(const ListArgs& a, int n_sm, cudaStream_t s) {
    const int64_t blocks = (a.n + kRowWarps - 1) / kRowWarps, most = short_ctas<T, kOp, N, kLong>() * (int64_t)n_sm;
    return launch_after(token_list_short_kernel<T, kOp, N, kLong>, (unsigned)(blocks < most ? blocks : most), 32 * kRowWarps, 0, s, a);
}
// nv: most vectors of a row, 256 at most.
template <class T, int kOp>
cudaError_t launch_list_short(const ListArgs& a, int64_t nv, int n_sm, cudaStream_t s) {
    if constexpr (kOp != kListDrawAll) {
        if (a.K > kShortTop && nv > 64) return launch_list_short_as<T, kOp, 8, true>(a, n_sm, s);
        if (a.K > kShortTop) return launch_list_short_as<T, kOp, 2, true>(a, n_sm, s);
    }
    if (nv <= 32) return launch_list_short_as<T, kOp, 1, false>(a, n_sm, s);
    if (nv <= 64) return launch_list_short_as<T, kOp, 2, false>(a, n_sm, s);
    if (nv <= 128) return launch_list_short_as<T, kOp, 4, false>(a, n_sm, s);
    return launch_list_short_as<T, kOp, 8, false>(a, n_sm, s);
}

}  // namespace

}  // namespace malib
