// Token policies, the rollout's side: a row's most likely entries and the draw of its token.
// A row holds logits z_0 .. z_{V-1}; its entries are in the order of falling z, the lower index
// first among equal ones (-0 equals 0). With the row's statistics (m, S, t) as for the losses,
// ln p_j = (z_j - m) / T - ln S, and the order of z is that of p. A masked entry (-infinity) is
// never listed and never drawn.
//
// The first K entries: an entry's key is its logit's bits, mapped so that larger logits have
// larger keys, with the index below them, so that no two keys are equal (56 bits). A bound is
// looked for with at least K keys and at most kListCap above it; what lies above it is collected,
// sorted, and cut at K. The bound comes from the maxima of groups of entries, which the
// statistics' pass leaves: the K-th largest maximum has at least K entries above it, and as few
// more as groups have several of the first entries. Only the groups whose maximum reaches it are
// read again. The maxima's keys are held in 16 bits, which lowers the bound to the next
// such value; which one that is, a histogram of their distances from the row's maximum says.
// Where that leaves more than kListCap entries (many equal ones, or the first entries in
// few groups), the bound is found from all keys: a histogram of their top 8 bits says in which bin
// the K-th lies, one of the next 8 bits looks into that bin, and so on.
//
// The draw from the whole row takes the entries in the order of their index: sums of segments of 256
// vectors are kept from the statistics' pass, the one that holds u times the whole is found among
// them, and its entries alone are read again. The draw from a list takes them in the list's order.
// A row's token is the same whatever its batch: neither the CTAs that share the row nor its place in memory
// change a sum that decides it. Segments and their vectors are counted from the row's first entry (a vector
// that the memory does not have so is put together from two), a segment's sum is relative to its own maximum,
// and the segments are added in their order by one warp. (Segments of the memory's vectors, relative to the
// maximum so far, gave 14 of 3,000 draws from 131,072 bf16 entries another token by a cluster than by the stream.)
//
// Rows of more than 4 KB (shorter ones: token_list_short.cuh) are a block's of 64, 128 or 256 threads each, or a
// cluster's. The floor is reading the row once. What bounds it: a block's loads, none of which are in flight while
// the batch before is summed (the sums alone run at 4.9 TB/s so, at 6.4 as a stream), the instructions of the sums (some
// six an entry), and a row's selection, a chain of a dozen short steps with barriers between them that takes half as
// long again: the blocks of an SM are at different steps. 8,192 x 65,536 bf16, a quarter left out, 64 entries
// 180 us (4.5 TB/s, issue slots 60 %), 4,096 draws from the first 50 of 32,768 62 us (3.9 TB/s, 53 %), 333 x 151,111
// fp32 with 1,024 80 us; one row of 131,072 with 20 by eight CTAs 10. Prefetches of the next batches into
// L2 cost 6 %.
#pragma once

#include <cfloat>
#include <type_traits>

#include "token_common.cuh"
#include "token_peer.cuh"
#include "token_rollout.h"
#include "token_shift.cuh"

namespace malib {

struct ListShape {
    int cluster, slice;                              // CTAs a row, vectors of a CTA's slice
    int group_log;                                   // log 2 of a maximum's vectors; < 0: no maxima
    int cap;                                         // most keys that are sorted
    int room;                                        // sorted keys, or twice as many groups to be read again
    int maxima;                                      // bytes of the groups' maxima
    int slice_K;                                     // entries that a CTA lists: K, or a share of it
};

namespace {

constexpr int kListCap = 2048;                       // most keys that are sorted, for any list
constexpr int kListMost = 160 << 10;                 // dynamic shared memory: segments of 2^24 fp32 entries take 131 KB
constexpr int kListPer = 8;                          // vectors of a thread in a batch
constexpr int kWordVecs = 4, kWords = kListPer / kWordVecs;          // of a word of maxima; words of a batch
constexpr int kListBins = 1024;                      // of the maxima's distances
constexpr int kListGroups = 16384;                   // most maxima of a slice
constexpr uint32_t kIndexMask = (1u << 24) - 1;

// Larger for larger logits; the same for -0 and 0.
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __float_as_uint(__fadd_rn(z, 0.f));
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ uint64_t entry_key(float z, int j) {
    return (uint64_t)order_key(z) << 24 | (kIndexMask - (uint32_t)j);
}
__device__ __forceinline__ int key_index(uint64_t key) { return (int)(kIndexMask - ((uint32_t)key & kIndexMask)); }
__device__ __forceinline__ float key_logit(uint64_t key) { return order_value((uint32_t)(key >> 24)); }

// What a CTA's peers take from it.
struct __align__(16) ListShared {
    float4 stat;                                     // m, S, t, entries before the token (bits)
    uint32_t count;                                  // keys collected; past the cap: not all are there
    uint32_t reach;                                  // the top 16 bits from which on they are all; 0: all are
    uint32_t pad[2];
    uint32_t hist[kListBins];                        // or two of 256 bins
};
struct ListPick {
    uint32_t digit, above, at;                       // of a histogram; at = 0: fewer than K entries in all
};

// The largest of each group of 1, 2, 4 or 8 vectors, as the top 16 bits of its key, to out[0], out[stride] ..; 0:
// none. Larger groups are their caller's. What comes back is the largest of all.
__device__ __forceinline__ uint16_t max_key(float z) { return z > -INFINITY ? (uint16_t)(order_key(z) >> 16) : (uint16_t)0; }
template <class T>
__device__ __forceinline__ float group_maxima(const uint4 (&x)[kListPer], int group_log, uint16_t* out, int stride) {
    uint32_t m[kListPer];
#pragma unroll
    for (int u = 0; u < kListPer; ++u)
        m[u] = Elt<T>::max(Elt<T>::max(x[u].x, x[u].y), Elt<T>::max(x[u].z, x[u].w));
#pragma unroll
    for (int n = kListPer; n > 0; n /= 2) {
        if (n << group_log == kListPer)
#pragma unroll
            for (int i = 0; i < n; ++i) out[i * stride] = max_key(Elt<T>::largest(m[i]));
#pragma unroll
        for (int i = 0; i < n / 2; ++i) m[i] = Elt<T>::max(m[2 * i], m[2 * i + 1]);
    }
    return Elt<T>::largest(m[0]);
}

template <class T>
struct RowView {
    const T* z;
    int h, nv, V;                                    // entries before the first in its vector; vectors
    __device__ __forceinline__ uint4 vec(int v) const {
        const int j = v * Elt<T>::W - h;
        return j >= 0 && j + Elt<T>::W <= V ? *reinterpret_cast<const uint4*>(z + j) : load_part(z, j, V);
    }
};
template <class T>
__device__ __forceinline__ float entry_of(const uint4& q, int i) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    return Elt<T>::get(Elt<T>::word(w, i));
}
// A row's vectors by the index of their entries, wherever it lies in memory: v holds entries v W .. v W + W - 1 and
// is put together from the memory's vectors v and v + 1 where the row starts inside one.
template <int kWord>
struct Word {
    static constexpr int at = kWord;
};
// f(Word<the word of a vector that the row's entries start in>).
template <class F>
__device__ __forceinline__ void by_word(int by, F f) {
    if (by < 8) {                                    // (a switch would look its way up in memory)
        if (by < 4) f(Word<0>{});
        else f(Word<1>{});
    } else {
        if (by < 12) f(Word<2>{});
        else f(Word<3>{});
    }
}
// A warp's vectors of the memory, lane + 32 u of them in lane `lane`, to as many of the row that starts `by` bytes
// inside a vector. after: in lane 0, the vector behind the last.
template <class T, int N>
__device__ __forceinline__ void realign(uint4 (&x)[N], const uint4& after, int by, int lane) {
    const uint32_t bits = 8u * (by & 3);
    by_word(by, [&](auto word) {
        constexpr int k = decltype(word)::at;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const uint4 next = u + 1 < N ? x[u + 1 < N ? u + 1 : u] : after;
            const uint32_t mine[4] = {x[u].x, x[u].y, x[u].z, x[u].w}, his[4] = {next.x, next.y, next.z, next.w};
            uint32_t b[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < (sizeof(T) == 4 ? k : k + 1); ++i)
                b[i] = __shfl_sync(0xffffffffu, lane == 0 ? his[i] : mine[i], (lane + 1) & 31);
            x[u] = shifted<k>(x[u], make_uint4(b[0], b[1], b[2], b[3]), bits);
        }
    });
}
template <class T>
struct IndexView {
    static constexpr int W = Elt<T>::W;
    const T* z;
    int V;
    __device__ __forceinline__ int vectors() const { return (V + W - 1) / W; }
    __device__ __forceinline__ uint4 vec(int v) const {
        const int by = (int)((uintptr_t)z & 15u), h = by / (int)sizeof(T), j = v * W;
        if (by == 0 ? j + W > V : j < h || j - h + 2 * W > V) return load_part(z, j, V);
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(z + j) - by);
        if (by == 0) return *p;
        uint4 r;
        by_word(by, [&](auto word) { r = shifted<decltype(word)::at>(p[0], p[1], 8u * (by & 3)); });
        return r;
    }
};
// f(j, z) for the unmasked entries of vectors [v0, v1), by n threads.
template <class T, class F>
__device__ __forceinline__ void each_entry(const RowView<T>& r, int v0, int v1, int tid, int n, F f) {
    for (int v = v0 + tid; v < v1; v += n) {
        const uint4 q = r.vec(v);
#pragma unroll
        for (int i = 0; i < Elt<T>::W; ++i) {
            const float z = entry_of<T>(q, i);
            if (z > -INFINITY) f(v * Elt<T>::W - r.h + i, z);
        }
    }
}

// How many entries of vectors are >= a threshold (twice in a word for 16-bit types): at most 65,535 in a
// row between two calls of take().
template <class T>
struct Above;
template <>
struct Above<float> {
    uint32_t n = 0;
    __device__ static float next(float z) {          // the smallest larger value
        return order_value(order_key(z) + 1);
    }
    __device__ static uint32_t both(float z) { return __float_as_uint(z); }
    __device__ __forceinline__ void add(const uint4& q, uint32_t thr) {
        n += mask(q.x, thr) + mask(q.y, thr);
        n += mask(q.z, thr) + mask(q.w, thr);
    }
    __device__ __forceinline__ uint32_t take() {
        const uint32_t r = 0u - n;
        n = 0;
        return r;
    }
    __device__ static uint32_t mask(uint32_t z, uint32_t thr) {      // -1 or 0
        uint32_t r;
        asm("set.ge.u32.f32 %0, %1, %2;" : "=r"(r) : "f"(__uint_as_float(z)), "f"(__uint_as_float(thr)));
        return r;
    }
};
// The 16-bit value after z's in the order of the values.
__device__ __forceinline__ uint16_t next_half(uint16_t b) {
    if (b == 0x8000u) b = 0;                         // -0 is 0
    return b & 0x8000u ? (b == 0x8001u ? 0x8000u : b - 1) : b + 1;
}
// Comparisons of two give a word of two masks; masks are -1 in their half, and their sum's low half
// borrows from the high one.
__device__ __forceinline__ uint32_t count_masks(uint32_t sum) {
    const uint32_t lo = (0u - sum) & 0xffffu;
    return 2 * lo - ((sum + lo) >> 16 & 0xffffu) & 0xffffu;
}
template <>
struct Above<__nv_bfloat16> {
    uint32_t n = 0;
    __device__ static float next(float z) {
        return __bfloat162float(__ushort_as_bfloat16(next_half(__bfloat16_as_ushort(__float2bfloat16_rn(z)))));
    }
    __device__ static uint32_t both(float z) { return __bfloat16_as_ushort(__float2bfloat16_rn(z)) * 0x10001u; }
    __device__ __forceinline__ void add(const uint4& q, uint32_t thr) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) n += mask(w[i], thr);
    }
    __device__ static uint32_t mask(uint32_t z, uint32_t thr) {      // -1 or 0 in each half
        __nv_bfloat162 v, t;
        *reinterpret_cast<uint32_t*>(&v) = z;
        *reinterpret_cast<uint32_t*>(&t) = thr;
        return __hge2_mask(v, t);
    }
    __device__ __forceinline__ uint32_t take() {
        const uint32_t r = count_masks(n);
        n = 0;
        return r;
    }
};
template <>
struct Above<__half> {
    uint32_t n = 0;
    __device__ static float next(float z) {
        return __half2float(__ushort_as_half(next_half(__half_as_ushort(__float2half_rn(z)))));
    }
    __device__ static uint32_t both(float z) { return __half_as_ushort(__float2half_rn(z)) * 0x10001u; }
    __device__ __forceinline__ void add(const uint4& q, uint32_t thr) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) n += mask(w[i], thr);
    }
    __device__ static uint32_t mask(uint32_t z, uint32_t thr) {
        __half2 v, t;
        *reinterpret_cast<uint32_t*>(&v) = z;
        *reinterpret_cast<uint32_t*>(&t) = thr;
        return __hge2_mask(v, t);
    }
    __device__ __forceinline__ uint32_t take() {
        const uint32_t r = count_masks(n);
        n = 0;
        return r;
    }
};

// Sorts the n keys at `key` (room for the next power of two, 512 at least), largest first; what comes back
// has the first K in order, n how many are left. Few of them are counted: a key's place is how many are
// larger; several lanes
// share a key's count. narrow: bf16 logits, whose keys have 16 bits, and indexes below 2^16: 32 bits hold both.
// buckets: what the sort of more keys by bins needs.
struct Buckets {
    uint32_t top_key;                                // of the row's maximum, 32 bits
    uint32_t *bins, *warp_total;                     // [kListBins], [warps]
    uint16_t* order;                                 // [cap]
};
template <int kThreads, class Sync>
__device__ __forceinline__ const uint64_t* sort_keys(uint64_t* key, uint64_t* sorted, int& n, int K, bool narrow, int tid,
                                                     Sync sync, const Buckets& buckets) {
    const int enough = K + K / 4 + 12;
    if (n > 96 && n > enough + 32 && n <= 2 * kThreads) {
        // Fewer of them: a bound that at least K reach is bisected among the logits' bits, each thread with two
        // keys. (54 x 151,120 bf16 with 56 entries by four CTAs: 21.8 us with all counted against all, 16.6.)
        uint64_t own[2];
        uint32_t bits[2], lo = ~0u, hi = buckets.top_key + 1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            own[i] = tid + i * kThreads < n ? key[tid + i * kThreads] : 0ull;
            bits[i] = (uint32_t)(own[i] >> 24);
            if (own[i] != 0) lo = min(lo, bits[i]);
        }
        lo = __reduce_min_sync(0xffffffffu, lo);
        if ((tid & 31) == 0) buckets.warp_total[tid >> 5] = lo;
        sync();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) lo = min(lo, buckets.warp_total[w]);
        while (n > enough && hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            const int c = __syncthreads_count(bits[0] >= mid) + __syncthreads_count(bits[1] >= mid);
            if (c >= K) {
                lo = mid;
                n = c;
            } else {
                hi = mid;
            }
        }
        sync();
        if (tid == 0) buckets.warp_total[0] = 0;
        sync();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (own[i] != 0 && bits[i] >= lo) key[atomicAdd(buckets.warp_total, 1u)] = own[i];
        sync();
    }
    if (n <= max(128, kThreads + kThreads / 2)) {
        const int lanes = n * 8 <= kThreads ? 8 : n * 4 <= kThreads ? 4 : n * 2 <= kThreads ? 2 : 1;
        const auto narrowed = [](uint64_t k) { return (uint32_t)(k >> 24) & 0xffff0000u | (uint32_t)k & 0xffffu; };
        narrow = narrow && n <= 256;
        uint32_t* low = reinterpret_cast<uint32_t*>(key + 256);
        if (narrow) {
            for (int i = tid; i < (n + 3) / 4 * 4; i += kThreads) low[i] = i < n ? narrowed(key[i]) : 0u;
        } else if (tid == 0 && n % 2 != 0) {
            key[n] = 0ull;
        }
        sync();
        const int vecs = narrow ? (n + 3) / 4 : (n + 1) / 2;
        const uint4* quad = reinterpret_cast<const uint4*>(low);
        const ulonglong2* pair = reinterpret_cast<const ulonglong2*>(key);
        for (int i0 = 0; i0 < n; i0 += kThreads / lanes) {           // (the same rounds in every thread)
            const int i = i0 + tid / lanes;
            if (__all_sync(0xffffffffu, i >= n)) continue;
            const uint64_t own = i < n ? key[i] : ~0ull;
            int place = 0;
            if (narrow) {
                const uint32_t own_low = narrowed(own);
#pragma unroll 2
                for (int j = tid & (lanes - 1); j < vecs; j += lanes) {
                    const uint4 q = quad[j];
                    place += q.x > own_low;
                    place += q.y > own_low;
                    place += q.z > own_low;
                    place += q.w > own_low;
                }
            } else {
#pragma unroll 2
                for (int j = tid & (lanes - 1); j < vecs; j += lanes) {
                    const ulonglong2 q = pair[j];
                    place += q.x > own;
                    place += q.y > own;
                }
            }
            for (int o = lanes / 2; o > 0; o /= 2) place += __shfl_xor_sync(0xffffffffu, place, o);
            if (i < n && (tid & (lanes - 1)) == 0 && place < K) sorted[place] = own;
        }
        sync();
        return sorted;
    }
    const uint32_t top_key = buckets.top_key;
    uint32_t *bins = buckets.bins, *warp_total = buckets.warp_total;
    uint16_t* order = buckets.order;
    // More of them, by the distance of a key's logit from the row's maximum, in 1,024 equal steps of the
    // logits' bits: a key comes after those of smaller distances, and is counted among its bin's.
    // Bins of many keys are left to the sort below.
    constexpr int kBins = kListBins / kThreads;
    const int lane = tid & 31, warp = tid >> 5;
    uint32_t least = ~0u;
    for (int i = tid; i < n; i += kThreads) least = min(least, (uint32_t)(key[i] >> 24));
    least = __reduce_min_sync(0xffffffffu, least);
    if (lane == 0) warp_total[warp] = least;
    sync();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) least = min(least, warp_total[w]);
    const int shift = max(0, 22 - __clz(top_key - least));       // distances below 2^(10 + shift)
    const auto bin_of = [&](uint64_t k) { return (top_key - (uint32_t)(k >> 24)) >> shift; };
    for (int i = tid; i < kListBins; i += kThreads) bins[i] = 0;
    sync();
    for (int i = tid; i < n; i += kThreads) atomicAdd(bins + bin_of(key[i]), 1u);
    sync();
    uint32_t sum = 0, most = 0, size[kBins];
#pragma unroll
    for (int i = 0; i < kBins; ++i) {
        size[i] = bins[kBins * tid + i];
        sum += size[i];
        most = max(most, size[i]);
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t q = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += q;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) warp_total[warp] = upto | (most > 256 ? 1u << 31 : 0u);
    sync();
    bool many = false;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        const uint32_t q = warp_total[w];
        many |= q >> 31;
        if (w < warp) upto += q & 0x7fffffffu;
    }
    if (!many) {
        // a bin's first place, then, when its keys have taken theirs, the next bin's
        upto -= sum;
#pragma unroll
        for (int i = 0; i < kBins; ++i) {
            bins[kBins * tid + i] = upto;
            upto += size[i];
        }
        sync();
        for (int i = tid; i < n; i += kThreads) order[atomicAdd(bins + bin_of(key[i]), 1u)] = (uint16_t)i;
        sync();
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t own = key[i];
            const uint32_t bin = bin_of(own), first = bin > 0 ? bins[bin - 1] : 0u, end = bins[bin];
            int place = (int)first;
            if (place >= K) continue;
            for (uint32_t o = first; o < end; ++o) place += key[order[o]] > own;
            if (place < K) sorted[place] = own;
        }
        sync();
        return sorted;
    }
    int P = 256;
    while (P < n) P *= 2;
    for (int i = n + tid; i < P; i += kThreads) key[i] = 0ull;
    sync();
    for (int size = 2; size <= P; size *= 2)
        for (int gap = size / 2; gap > 0; gap /= 2) {
            for (int i = tid; i < P / 2; i += kThreads) {
                const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
                const uint64_t x = key[lo], y = key[hi];
                if ((x < y) == ((lo & size) == 0)) {
                    key[lo] = y;
                    key[hi] = x;
                }
            }
            sync();
        }
    return key;
}

__device__ __forceinline__ float warp_scan(float v, int lane) {      // inclusive
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const float b = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += b;
    }
    return v;
}
__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// A row's random number in [0, 1), infinity for what draws the last entry: what is read for it, and the number.
struct RowUniform {
    float u;
    uint32_t step;
    uint64_t sequence;
};
__device__ __forceinline__ RowUniform load_uniform(const ListArgs& a, int64_t row) {
    if (a.uniform) return RowUniform{a.uniform[row], 0u, 0ull};
    return RowUniform{0.f, (uint32_t)a.step[row], (uint64_t)a.sequence[row]};
}
__device__ __forceinline__ float uniform_of(const ListArgs& a, const RowUniform& r) {
    if (a.uniform) return r.u < 1.f ? r.u : INFINITY;
    return u24(draw(r.sequence, r.step, a.agent, a.seed).x);
}
__device__ __forceinline__ float row_uniform(const ListArgs& a, int64_t row) {
    if (a.uniform) {
        const float u = a.uniform[row];
        return u < 1.f ? u : INFINITY;
    }
    return u24(draw((uint64_t)a.sequence[row], (uint32_t)a.step[row], a.agent, a.seed).x);
}

__device__ __forceinline__ void write_draw(const ListArgs& a, int64_t row, int token, float logp, float H, float drawn) {
    if (a.drawn) a.drawn[row] = token;
    if (a.logp) a.logp[row] = logp;
    if (a.entropy) a.entropy[row] = H;
    if (a.draw_logp) a.draw_logp[row] = drawn;
}

// The draw from a sorted list (one warp). w_i = 2^x_i; kept are the entries before which less than
// top_p of the list's mass lies; the token is the first whose running mass exceeds u times the kept
// one.
__device__ __forceinline__ void draw_listed(const ListArgs& a, int64_t row, const RowStat& r, const uint64_t* key, int n,
                                            int lane) {
    const int per = (n + 31) / 32, i0 = min(n, lane * per), i1 = min(n, i0 + per);
    float own = 0.f;
    for (int i = i0; i < i1; ++i) own += exp2_fast(x_of(key_logit(key[i]), r.m, a.k));
    const float before = warp_scan(own, lane) - own, total = __shfl_sync(0xffffffffu, before + own, 31);
    // the kept ones' number, mass, and sum of w x
    float cum = before, mass = 0.f, t = 0.f;
    int kept = 0;
    for (int i = i0; i < i1; ++i) {
        if (i > 0 && a.top_p < 1.f && !(cum < a.top_p * total)) break;
        const float x = x_of(key_logit(key[i]), r.m, a.k), w = exp2_fast(x);
        cum += w;
        mass = cum;
        t = fmaf(w, fmaxf(x, kXMin), t);
        kept = i + 1;
    }
    mass = warp_max(mass);
    t = warp_add(t);
    kept = __reduce_max_sync(0xffffffffu, kept);
    const float target = row_uniform(a, row) * mass;
    int at = -1, last = -1;
    cum = before;
    for (int i = i0; i < min(i1, kept); ++i) {
        const float w = exp2_fast(x_of(key_logit(key[i]), r.m, a.k));
        cum += w;
        if (w > 0.f) last = i;
        if (at < 0 && w > 0.f && cum > target) at = i;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, at >= 0);
    at = hit ? __shfl_sync(0xffffffffu, at, __ffs(hit) - 1) : __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) {
        const float z = key_logit(key[at]);
        write_draw(a, row, key_index(key[at]), log_prob(a, r, z), row_entropy(r), log_prob(a, RowStat{r.m, mass, t}, z));
    }
}

// The draw from a whole row (one warp): the segment that holds the target, then its entries. A lane has a segment,
// or of more than 32 an odd number of them that follow one another; of more than 256 the lanes' masses are added
// in 64 bits. Where rounding leaves no entry, the last one that has a mass is drawn. (No product here may join an
// addition: the compiler would be free to round one caller's differently. Loops, not unrolled ones: a warp goes
// through this once a row, and what it takes is mostly the instructions' way to it.)
// An entry's mass is 0 below 2^-126 of the largest, but a sum of such entries, relative to a smaller
// maximum, need not be: a segment (2,048 entries at most) counts from 2^-112 on, so that it has an entry that does.
constexpr int kSegmentVecs = 32 * kListPer;
constexpr float kSegmentLeast = 0x1p-112f;
__device__ __forceinline__ double warp_scan(double v, int lane) {
#pragma unroll 1
    for (int o = 1; o < 32; o *= 2) {
        const double b = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += b;
    }
    return v;
}
// The first of the lanes that passes the target, or the last that has a mass.
__device__ __forceinline__ int pick_lane(bool over, bool some, bool& hit) {
    const unsigned o = __ballot_sync(0xffffffffu, over), s = __ballot_sync(0xffffffffu, some);
    hit = o != 0;
    return o ? __ffs(o) - 1 : 31 - __clz(s | 1u);
}
// The segment that holds u times the whole; rest: that less the mass before it. mass(i, have): of segment i, 0 if not.
template <class Sum, class Mass>
__device__ __forceinline__ int find_segment(int segments, float u01, Mass mass, float& rest, int lane) {
    const int of = segments <= 32 ? 1 : (segments + 31) / 32 | 1;    // of a lane
    Sum w;
    if constexpr (sizeof(Sum) == 4) {
        w = mass(lane * of, true);
#pragma unroll 1
        for (int i = 1; i < of; ++i) w += mass(lane * of + i, true);
    } else {
        Sum2 sum{0.f, 0.f};
#pragma unroll 4
        for (int i = 0; i < of; ++i) sum.add(mass(lane * of + i, true));
        w = (double)sum.s + (double)sum.e;
    }
    const Sum cum = warp_scan(w, lane), total = __shfl_sync(0xffffffffu, cum, 31);
    Sum target;
    if constexpr (sizeof(Sum) == 4) target = __fmul_rn(u01, total);
    else target = __dmul_rn((double)u01, total);
    bool hit;
    const int group = pick_lane(w > 0 && cum > target, w > 0, hit);
    rest = (float)(target - __shfl_sync(0xffffffffu, cum - w, group));
    if (of == 1) return group;
    float passed = 0.f, before = 0.f;
    int at = 0;
    hit = false;
#pragma unroll 1
    for (int i = 0; i < of && !hit; i += 32) {
        const float v = mass(group * of + i + lane, i + lane < of), upto = warp_scan(v, lane);
        const int k = pick_lane(v > 0.f && passed + upto > rest, v > 0.f, hit);
        if (__shfl_sync(0xffffffffu, v, k) > 0.f) {
            at = group * of + i + k;
            before = passed + __shfl_sync(0xffffffffu, upto - v, k);
        }
        passed += __shfl_sync(0xffffffffu, upto, 31);
    }
    rest -= before;
    return at;
}
// here(i): whether this warp finds the entry of segment i (CTAs of a cluster have their own).
template <class T, class Here>
__device__ __forceinline__ void draw_all(const ListArgs& a, int64_t row, const RowStat& r, const IndexView<T>& view,
                                         const float2* segment, float u01, Here here, int lane) {
    constexpr int W = Elt<T>::W;
    const int segments = (view.vectors() + kSegmentVecs - 1) / kSegmentVecs;
    const auto mass = [&](int i, bool have) {
        const float2 sg = have && i < segments ? segment[i] : make_float2(-INFINITY, 0.f);
        const float w = sg.y > 0.f ? __fmul_rn(sg.y, exp2_fast(fmaxf((sg.x - r.m) * a.k, kXMin) + kExpBias)) : 0.f;
        return w < kSegmentLeast ? 0.f : w;
    };
    float rest;
    const int at = segments <= 256 ? find_segment<float>(segments, u01, mass, rest, lane)
                                   : find_segment<double>(segments, u01, mass, rest, lane);
    if (!here(at)) return;
    const int v0 = at * kSegmentVecs + lane, v_hi = view.vectors();
    float sum = 0.f, fz = 0.f, bz = 0.f;
    int found = -1, behind = -1;                     // the entry that passes the target; the last one with a mass
#pragma unroll 1
    for (int u = 0; u < kListPer && !__any_sync(0xffffffffu, found >= 0); ++u) {
        const int v = v0 + u * 32;
        const uint4 q = v < v_hi ? view.vec(v) : Elt<T>::none();
        float e[W], mine = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            e[i] = exp2_fast(x_of(entry_of<T>(q, i), r.m, a.k));
            mine += e[i];
        }
        const float incl = warp_scan(mine, lane);
        float cum = sum + (incl - mine);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            cum += e[i];
            if (e[i] > 0.f && found < 0) {
                behind = v * W + i;
                bz = entry_of<T>(q, i);
                if (cum > rest) {
                    found = behind;
                    fz = bz;
                }
            }
        }
        sum += __shfl_sync(0xffffffffu, incl, 31);
    }
    const unsigned at_hit = __ballot_sync(0xffffffffu, found >= 0);
    int lane_at = __ffs(at_hit) - 1;
    if (!at_hit) {
        lane_at = __ffs(__ballot_sync(0xffffffffu, behind == __reduce_max_sync(0xffffffffu, behind))) - 1;
        found = behind;
        fz = bz;
    }
    if (lane == lane_at) {
        const float logp = log_prob(a, r, fz);
        write_draw(a, row, found, logp, row_entropy(r), logp);
    }
}

// A key with at least K keys from it on, or 0 where there are fewer, and at most `cap`: by the keys'
// digits of 8 bits. bins: two histograms; meet: every CTA of the row is there; total: a bin of
// all of them.
template <class T, int kThreads, class Sync, class Meet, class Total>
__device__ __forceinline__ uint64_t bound_of_all(const RowView<T>& view, int v_lo, int v_hi, uint32_t K, uint32_t cap,
                                                 uint32_t* bins, ListPick* pick, int tid, Sync sync, Meet meet, Total total) {
    uint64_t bound = 0;
    uint32_t above = 0;
    int shift = 48;
    for (int pass = 0;; ++pass, shift -= 8) {
        uint32_t* hist = bins + 256 * (pass & 1);
        for (int i = tid; i < 256; i += kThreads) hist[i] = 0;
        sync();
        each_entry(view, v_lo, v_hi, tid, kThreads, [&](int j, float e) {
            const uint64_t key = entry_key(e, j);
            if (pass == 0 || key >> (shift + 8) == bound) atomicAdd(hist + ((uint32_t)(key >> shift) & 255u), 1u);
        });
        meet();
        if (tid < 32) {
            uint32_t n[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] = total(hist + (255 - 8 * tid - i));
                sum += n[i];
            }
            uint32_t upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
                if (tid >= o) upto += x;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, above + upto >= K);
            if (hit ? tid == __ffs(hit) - 1 : tid == 0) {
                ListPick p{0, 0, 0};
                uint32_t cum = above + upto - sum;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (hit && p.at == 0 && cum + n[i] >= K) p = ListPick{(uint32_t)(255 - 8 * tid - i), cum, n[i]};
                    cum += n[i];
                }
                *pick = p;
            }
        }
        sync();
        const ListPick p = *pick;
        if (p.at == 0) return 0;                     // in the first pass only
        bound = bound << 8 | p.digit;
        above = p.above;
        if (above + p.at <= cap) return bound << shift;
    }
}

// What a warp gathers a slice's statistics in: as for the losses' long rows, those of more than
// kManyBatches batches keep the errors of their parts' additions.
constexpr int kManyBatches = 16;
__device__ __forceinline__ void join(RowStat& r, const RowStat& part) {
    r.s += part.s;
    r.t += part.t;
}
__device__ __forceinline__ void join(LongStat& r, const RowStat& part) {
    r.s.add(part.s);
    r.t.add(part.t);
}

// The maxima of a thread's vectors, four of them to a word: of all 16 entries in 32 bits, of the 16 even and the
// 16 odd ones in 16 bits each.
template <class T>
struct Words {
    uint32_t w[kWords];
    float largest;
    __device__ __forceinline__ explicit Words(const uint4 (&x)[kListPer]) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
#pragma unroll
            for (int u = 0; u < kWordVecs; ++u) {
                const uint4& q = x[i * kWordVecs + u];
                const uint32_t v = Elt<T>::max(Elt<T>::max(q.x, q.y), Elt<T>::max(q.z, q.w));
                w[i] = u == 0 ? v : Elt<T>::max(w[i], v);
            }
            m = i == 0 ? w[i] : Elt<T>::max(m, w[i]);
        }
        largest = Elt<T>::largest(m);
    }
};

// Where z lies so far below the maximum that 2^x is 0, it is raised to a value there before it is widened, two
// entries at a time: x stays finite, and needs no bound of its own. low: that value in each half;
// 0: there is none (a temperature too large for the type, logits too large for fp32).
template <class T>
__device__ __forceinline__ uint32_t low_of(float m, float k, float reach) {
    return 0u;
}
__device__ __forceinline__ bool is_low(float low, float m, float k) {
    const float x = (low - m) * k;
    return x <= -150.f && x > -INFINITY;
}
template <>
__device__ __forceinline__ uint32_t low_of<__nv_bfloat16>(float m, float k, float reach) {
    const __nv_bfloat16 low = __float2bfloat16_rd(m - reach);
    return is_low(__bfloat162float(low), m, k) ? __bfloat16_as_ushort(low) * 0x10001u : 0u;
}
template <>
__device__ __forceinline__ uint32_t low_of<__half>(float m, float k, float reach) {
    const __half low = __float2half_rd(m - reach);
    return is_low(__half2float(low), m, k) ? __half_as_ushort(low) * 0x10001u : 0u;
}
// The two entries of a word less m.
template <class T>
__device__ __forceinline__ F2 word_less(uint32_t w, float m) {
    float a, b;
    if constexpr (std::is_same<T, __half>::value)
        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n sub.f32.f16 %0, l, %3;\n sub.f32.f16 %1, h, %3;\n}"
            : "=f"(a), "=f"(b) : "r"(w), "f"(m));
    else
        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n sub.f32.bf16 %0, l, %3;\n sub.f32.bf16 %1, h, %3;\n}"
            : "=f"(a), "=f"(b) : "r"(w), "f"(m));
    return f2_make(a, b);
}
// gather() of a part from 0, with `low` as above.
template <class T>
__device__ __forceinline__ RowStat gather_part(float m, const uint4 (&q)[kListPer], float k, uint32_t low) {
    RowStat r{m, 0.f, 0.f};
    if (sizeof(T) == 4 || low == 0u) {
        gather<T>(r, q, k);
        return r;
    }
    F2 s = 0ull, t = 0ull;
    const F2 k2 = f2_dup(k), bias = f2_dup(kExpBias);
#pragma unroll
    for (int u = 0; u < kListPer; ++u) {
        const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 x = f2_fma3(word_less<T>(Elt<T>::max(w[i], low), m), k2, bias), e = f2_exp2(x);
            s = f2_add(s, e);
            f2_fma(t, e, x);
        }
    }
    const float2 s2 = f2_split(s), t2 = f2_split(t);
    r.s = s2.x + s2.y;
    r.t = t2.x + t2.y;
    return r;
}

// A draw's segment: its sums are relative to its own maximum mx (a warp's lanes have the same), and join those
// of the segments so far relative to theirs. What comes back is the warp's whole mass.
template <class T, class Own>
__device__ __forceinline__ float sum_segment(Own& st, const uint4 (&x)[kListPer], float mx, float k, float low_reach) {
    if (!(mx <= st.m)) raise(st, mx, k);
    RowStat part{mx, 0.f, 0.f};
    if (mx != -INFINITY) part = gather_part<T>(mx, x, k, low_of<T>(mx, k, low_reach));
    const float s = warp_add(part.s);
    if (mx < st.m) {
        const float d = fmaxf((mx - st.m) * k, kXMin), f = exp2_fast(d + kExpBias);
        part.t = f * fmaf(part.s, d, part.t);
        part.s *= f;
    }
    join(st, part);
    return s;
}

// How a slice's statistics and maxima are held. kCoarse: words of maxima, and the bound from the
// threads' own maxima, of which there are two for every entry of the list; kWide: from the words', of
// which there are four; kFine: finer groups, and the bound from theirs. kLong: more than kManyBatches
// batches, any groups. kEntries: no groups; all entries are sorted, or where they are too many the
// bound comes from theirs.
enum : int { kCoarse = 0, kFine = 1, kLong = 2, kEntries = 3, kWide = 4 };
template <int kMode>
struct OwnStat {
    using Type = RowStat;
};
template <>
struct OwnStat<kLong> {
    using Type = LongStat;
};

template <class T, int kOp, int kThreads, int kMode>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? (kOp == kListDrawAll ? 3 : 4) : kThreads == 128 ? 7 : 14) token_list_kernel(ListArgs a, ListShape sh) {
    using Own = typename OwnStat<kMode>::Type;
    constexpr int W = Elt<T>::W, kWarps = kThreads / 32, kWarpVecs = kSegmentVecs, kBatch = kWarps * kWarpVecs;
    constexpr bool kAll = kOp == kListDrawAll, kWordMaxima = kMode == kCoarse || kMode == kWide;
    // keys [cap], sorted ones [room] (or groups to be read again), maxima; or segments' (m, S)
    extern __shared__ __align__(16) uint64_t keys[];
    __shared__ ListShared own;
    __shared__ float4 red[kWarps], peers[kAll ? 8 : 1];              // peers: the statistics of a draw's CTAs
    __shared__ ListPick pick;
    __shared__ uint32_t n_again, warp_total[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = sh.cluster, rank = C > 1 ? (int)cluster_rank() : 0;
    uint64_t* sorted = keys + sh.cap;
    uint32_t* again = reinterpret_cast<uint32_t*>(sorted);
    uint16_t* maxima = reinterpret_cast<uint16_t*>(sorted + sh.room);
    uint32_t* words = reinterpret_cast<uint32_t*>(sorted + sh.room);         // kCoarse: [batch][word][thread]
    uint16_t* order = reinterpret_cast<uint16_t*>(reinterpret_cast<uint8_t*>(maxima) + sh.maxima);
    float2* segment = reinterpret_cast<float2*>(keys);
    if (kAll && C > 1) cluster_arrive();
    wait_for_previous();
    let_next_start();
    // Every CTA of the row comes here; what each wrote before is seen by all after it.
    auto meet = [&] {
        if (C == 1) {
            __syncthreads();
        } else {
            cluster_arrive();
            cluster_wait();
        }
    };
    // The keys of a slice's entries that may be among the first K, those of the first K of the slice and
    // few more, to keys and their number to own.count (past the cap: not all are there). Every
    // thread of the block; r: the slice's statistics, maxima: those of its groups.
    auto collect = [&](const RowStat& r, const RowView<T>& view, int v_lo, int v_hi, float thread_max) {
        if (tid == 0) own.count = own.reach = n_again = pick.digit = 0;
        constexpr bool kGroups = kMode != kEntries;
        if (!kGroups && (v_hi - v_lo) * W <= sh.cap) {
            __syncthreads();
            each_entry(view, v_lo, v_hi, tid, kThreads, [&](int j, float e) {
                const uint32_t at = atomicAdd(&own.count, 1u);
                if (at < (uint32_t)sh.cap) keys[at] = entry_key(e, j);
            });
            __syncthreads();
            return;
        }
        const int log = kWordMaxima ? 2 : sh.group_log;         // of a group's vectors
        const int n_max = !kGroups ? 0 : (((v_hi - v_lo + kBatch - 1) / kBatch * kListPer + (1 << log) - 1) >> log) * kThreads;
        const uint32_t top_key = order_key(r.m) >> 16;
        uint32_t reach = 0;
        for (int coarse = 0; coarse <= 6 && reach == 0; coarse += 6) {       // bins of one value, then of 64
            constexpr int kBins = kListBins / kThreads;                      // of a thread
            uint4* bins = reinterpret_cast<uint4*>(own.hist + kBins * tid);
#pragma unroll
            for (int i = 0; i < kBins / 4; ++i) bins[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            const auto count = [&](uint32_t key) {
                const uint32_t bin = (top_key - key) >> coarse;
                if (key != 0 && bin < kListBins) atomicAdd(own.hist + bin, 1u);
            };
            if constexpr (!kGroups) each_entry(view, v_lo, v_hi, tid, kThreads, [&](int, float e) { count(max_key(e)); });
            else if constexpr (kMode == kCoarse) count(max_key(thread_max));
            else if constexpr (kMode == kWide)
                for (int i = tid; i < n_max; i += kThreads) count(max_key(Elt<T>::largest(words[i])));
            else
                for (int i = tid; i < n_max; i += kThreads) count(maxima[i]);
            __syncthreads();
            uint32_t sum = 0;
#pragma unroll
            for (int i = 0; i < kBins / 4; ++i) sum += (bins[i].x + bins[i].y) + (bins[i].z + bins[i].w);
            uint32_t upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t q = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += q;
            }
            if (lane == 31) warp_total[warp] = upto;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps - 1; ++w) upto += w < warp ? warp_total[w] : 0u;
            if (upto >= (uint32_t)sh.slice_K && upto - sum < (uint32_t)sh.slice_K) {
                uint32_t cum = upto - sum, bin = kBins * tid;
                while ((cum += own.hist[bin]) < (uint32_t)sh.slice_K) ++bin;
                // the bin's smallest value, at least 1 (0 has no entries)
                const uint32_t below = ((bin + 1) << coarse) - 1;
                pick.digit = below < top_key ? top_key - below : 1u;
            }
            __syncthreads();
            reach = pick.digit;
        }
        // (0: fewer than K groups have entries; all entries may be wanted)
        const uint32_t least = max(reach, 1u);
        if (tid == 0) own.reach = reach;
        // (a key below those of all values is a NaN's)
        const float smallest = reach > 0 ? fmaxf(order_value(reach << 16), -FLT_MAX) : -FLT_MAX;
        if constexpr (!kGroups) {                    // entries were counted themselves, not groups
            each_entry(view, v_lo, v_hi, tid, kThreads, [&](int j, float e) {
                if (!(e >= smallest)) return;
                const uint32_t at = atomicAdd(&own.count, 1u);
                if (at < (uint32_t)sh.cap) keys[at] = entry_key(e, j);
            });
            __syncthreads();
            return;
        }
        // (whole warps: n_max is a multiple of the block's threads)
        const auto push = [&](bool hit, int id, uint32_t& to) {
            const unsigned hits = __ballot_sync(0xffffffffu, hit);
            const uint32_t at = to + __popc(hits & ((1u << lane) - 1u));
            if (hit && at < 2u * sh.room) again[at] = id;
            to += __popc(hits);
        };
        const auto room_for = [&](bool first, bool second) {
            const int n = __popc(__ballot_sync(0xffffffffu, first)) + __popc(__ballot_sync(0xffffffffu, second));
            uint32_t to = 0;
            if (n > 0 && lane == 0) to = atomicAdd(&n_again, (uint32_t)n);
            return n > 0 ? __shfl_sync(0xffffffffu, to, 0) : ~0u;
        };
        if constexpr (kWordMaxima) {
            for (int i = tid; i < n_max; i += 2 * kThreads) {
                const bool x = Elt<T>::largest(words[i]) >= smallest, y = Elt<T>::largest(words[i + kThreads]) >= smallest;
                uint32_t to = room_for(x, y);
                if (to == ~0u) continue;
                push(x, i, to);
                push(y, i + kThreads, to);
            }
        } else {
            for (int i = tid; i < n_max; i += kThreads) {
                const bool x = maxima[i] >= least;
                uint32_t to = room_for(x, false);
                if (to != ~0u) push(x, i, to);
            }
        }
        __syncthreads();
        if (n_again > 2u * sh.room) {
            if (tid == 0) own.count = sh.cap + 1;
        } else {
            const int items = (int)n_again << log;
            constexpr int kAt = 2;                                           // loads in flight
            for (int i0 = tid; i0 < items; i0 += kAt * kThreads) {
                uint4 x[kAt];
                int v[kAt];
#pragma unroll
                for (int u = 0; u < kAt; ++u) {
                    const int item = i0 + u * kThreads;
                    x[u] = Elt<T>::none();
                    if (item >= items) continue;
                    const int id = (int)again[item >> log], n = (id / kThreads << log) + (item & ((1 << log) - 1));
                    v[u] = v_lo + (n >> 3) * kBatch + (id % kThreads >> 5) * kWarpVecs + (n & 7) * 32 + (id & 31);
                    if (v[u] < v_hi) x[u] = view.vec(v[u]);
                }
#pragma unroll
                for (int u = 0; u < kAt; ++u) {
                    if (!(vec_max<T>(reinterpret_cast<const uint4(&)[1]>(x[u])) >= smallest)) continue;
                    uint32_t hits = 0;
#pragma unroll
                    for (int i = 0; i < W; ++i) hits |= entry_of<T>(x[u], i) >= smallest ? 1u << i : 0u;
                    uint32_t to = atomicAdd(&own.count, (uint32_t)__popc(hits));
                    for (; hits; hits &= hits - 1, ++to) {
                        const int i = __ffs(hits) - 1;
                        float e = entry_of<T>(x[u], 0);
#pragma unroll
                        for (int o = 1; o < W; ++o)
                            if (i == o) e = entry_of<T>(x[u], o);
                        if (to < (uint32_t)sh.cap) keys[to] = entry_key(e, v[u] * W - view.h + i);
                    }
                }
            }
        }
        __syncthreads();
    };
    const float low_reach = 160.f / a.k;
    bool met = false;                                // the cluster's CTAs, at their start
    for (int64_t row = blockIdx.x / C; row < a.n; row += gridDim.x / C) {
        const int token = a.tokens ? a.tokens[row] : 0;
        const bool first = tid == 0 && rank == 0;
        bool live = token >= 0;
        if (kOp == kListTop && token >= a.V) {
            live = false;
            if (first) atomicOr(a.err, ERRBIT_BAD_TOKEN);
        }
        // (the same in every thread of the row's CTAs)
        auto no_list = [&](float logp) {
            if (kOp == kListTop && rank == 0)
                for (int i = tid; i < a.K; i += kThreads) {
                    a.top_ids[row * a.K + i] = -1;
                    a.top_logp[row * a.K + i] = logp;
                }
        };
        if (!live) {
            if (kOp == kListTop) {
                if (first) {
                    logp_row(a, row, false, RowStat{0.f, 1.f, 0.f}, 0.f);
                    if (a.rank) a.rank[row] = 0;
                }
                no_list(0.f);
            } else if (first) {
                write_draw(a, row, -1, 0.f, 0.f, 0.f);
            }
            continue;
        }
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
        const RowView<T> view{z, h, nv, a.V};
        const int v_lo = min(nv, rank * sh.slice), v_hi = min(nv, v_lo + sh.slice);
        float zt = 0.f;
        if (kOp == kListTop && a.tokens) zt = Elt<T>::get(z[token]);
        RowUniform random{};
        if (kAll && warp == 0) random = load_uniform(a, row);

        // ---- statistics; a warp's vectors of a batch follow one another
        Own st{};
        st.m = -INFINITY;
        uint32_t before = 0, low = 0;
        const bool ranked = kOp == kListTop && a.rank;
        Above<T> above;
        // entries count that are >= the token's before it, and larger ones behind it
        const uint32_t thr_before = ranked ? Above<T>::both(zt) : 0u, thr_behind = ranked ? Above<T>::both(Above<T>::next(zt)) : 0u;
        float thread_max = -INFINITY;                // of its vectors; kLong: of the present group's
        // the row's whole vectors; a partial first or last one is filled up
        const int full_lo = h > 0 ? 1 : 0, full_hi = (h + a.V) % W != 0 ? nv - 1 : nv;
        const uint4* src = reinterpret_cast<const uint4*>(z - h);
        const int per = sh.slice / kSegmentVecs;     // draws: segments of a CTA
        const int batches = (v_hi - v_lo + kBatch - 1) / kBatch;
        for (int batch = 0; batch < batches; ++batch) {
            const int b = v_lo + batch * kBatch, v0 = b + warp * kWarpVecs + lane;
            uint4 x[kListPer];
            if (b >= full_lo && b + kBatch <= min(v_hi, full_hi)) {
#pragma unroll
                for (int u = 0; u < kListPer; ++u) x[u] = src[v0 + u * 32];
            } else {
                const int n = max(0, min(v_hi, full_hi) - full_lo);
#pragma unroll
                for (int u = 0; u < kListPer; ++u)
                    x[u] = (uint32_t)(v0 + u * 32 - full_lo) < (uint32_t)n ? src[v0 + u * 32] : Elt<T>::none();
                if (v0 == 0 && full_lo > 0) x[0] = load_part(z, -h, a.V);
                const int tail = full_hi < nv && nv <= v_hi ? nv - 1 - v0 : -1;
                if (tail >= 0 && tail < kWarpVecs && tail % 32 == 0 && !(tail == 0 && v0 == 0 && full_lo > 0)) {
                    const uint4 q = load_part(z, (nv - 1) * W - h, a.V);
#pragma unroll
                    for (int u = 0; u < kListPer; ++u)
                        if (tail == u * 32) x[u] = q;
                }
            }
            if constexpr (kAll) {
                if (h > 0) {                         // (a slice's end is a batch's, or the row's)
                    const int next = v0 + kWarpVecs;
                    realign<T>(x, lane == 0 && next < nv ? view.vec(next) : Elt<T>::none(), (int)((uintptr_t)z & 15u), lane);
                }
            }
            float mx;
            if constexpr (kAll || kMode == kEntries) {
                mx = vec_max<T>(x);
            } else if constexpr (kWordMaxima) {
                const Words<T> m(x);
#pragma unroll
                for (int i = 0; i < kWords; ++i) words[(batch * kWords + i) * kThreads + tid] = m.w[i];
                mx = m.largest;
                thread_max = fmaxf(thread_max, mx);
            } else {
                mx = group_maxima<T>(x, sh.group_log, maxima + tid + (batch << 3 >> min(sh.group_log, 3)) * kThreads, kThreads);
                if (sh.group_log > 3) {
                    thread_max = fmaxf(thread_max, mx);
                    const int per = 1 << (sh.group_log - 3);
                    if ((batch + 1) % per == 0 || batch + 1 == batches) {
                        maxima[batch / per * kThreads + tid] = max_key(thread_max);
                        thread_max = -INFINITY;
                    }
                }
            }
            mx = warp_max(mx);
            if constexpr (kAll) {
                const float s = sum_segment<T>(st, x, mx, a.k, low_reach);
                // every CTA of the row has all segments
                float2* to = segment + (rank * per + batch * kWarps + warp);
                if (C == 1 && lane == 0) *to = make_float2(mx, s);
                if (C > 1) {
                    if (!met) cluster_wait();        // peers' shared memory is there to be written
                    met = true;
                    if (lane < C) peer_put(to, lane, make_float2(mx, s));
                }
                continue;
            }
            if (!(mx <= st.m)) {
                raise(st, mx, a.k);
                low = low_of<T>(st.m, a.k, low_reach);
            }
            RowStat part{st.m, 0.f, 0.f};
            if (st.m != -INFINITY) part = gather_part<T>(st.m, x, a.k, low);
            join(st, part);
            if (ranked && !(mx < zt)) {              // (a warp's entries are all before the token, behind it, or both)
                const int j0 = (v0 - lane) * W - h;
                if (j0 > token || j0 + kWarpVecs * W <= token) {
                    const uint32_t thr = j0 > token ? thr_behind : thr_before;
#pragma unroll
                    for (int u = 0; u < kListPer; ++u) above.add(x[u], thr);
                } else {
#pragma unroll
                    for (int u = 0; u < kListPer; ++u) above.add(x[u], (v0 + u * 32 + 1) * W - h <= token ? thr_before : thr_behind);
                }
                before += above.take();
            }
        }
        if (kAll && C > 1 && !met) cluster_wait();
        met = true;
        if (ranked) {
            // the token's own vector counted as one behind it; a masked token comes after every
            // entry before it
            if (zt == -INFINITY) {
                before = 0;
                if (first) before = (uint32_t)token;
                each_entry(view, max(v_lo, (token + h) / W), v_hi, tid, kThreads, [&](int j, float) { before += j >= token; });
            } else if (first) {
                for (int j = (token + h) / W * W - h; j < token; ++j) before += j >= 0 && Elt<T>::get(z[max(j, 0)]) == zt;
            }
        }
        RowStat r = stat_of(st);
        r.s = warp_add(r.s);
        r.t = warp_add(r.t);
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) red[warp] = make_float4(r.m, r.s, r.t, __uint_as_float(before));
        __syncthreads();
        {
            const float4 q = red[lane & (kWarps - 1)];
            r = reduce_stat<kWarps>(RowStat{q.x, q.y, q.z}, a.k);
            before = __reduce_add_sync(0xffffffffu, lane < kWarps ? __float_as_uint(q.w) : 0u);
        }
        // ---- the keys of the slice's first K entries, and what the peers take
        if constexpr (!kAll) {
            if (r.m != -INFINITY && fabsf(r.s) < INFINITY) collect(r, view, v_lo, v_hi, thread_max);
            else if (tid == 0) own.count = own.reach = 0;
        }
        float4 peer = make_float4(r.m, r.s, r.t, 0.f);               // lane i: CTA i's
        uint32_t n_keys = kAll ? 0 : own.count, reach = 0;
        if (C > 1) {
            if (kAll && warp == 0 && lane < C) peer_put(peers + rank, lane, peer);
            if (!kAll && tid == 0) own.stat = make_float4(r.m, r.s, r.t, __uint_as_float(before));
            meet();
            uint2 found = make_uint2(0u, 0u);        // (all loads before the first use)
            peer = make_float4(-INFINITY, 0.f, 0.f, 0.f);
            if (kAll && lane < C) peer = peers[lane];
            if (!kAll && lane < C) {
                peer = peer_load(&own.stat, lane);
                found = make_uint2(peer_load(&own.count, lane), peer_load(&own.reach, lane));
            }
            before = __reduce_add_sync(0xffffffffu, __float_as_uint(peer.w));
            r = reduce_stat<32>(RowStat{peer.x, peer.y, peer.z}, a.k);
            if (!kAll) {
                n_keys = __reduce_add_sync(0xffffffffu, found.x);
                reach = __reduce_max_sync(0xffffffffu, found.y);
            }
        }
        live = r.m != -INFINITY;
        const bool good = live && fabsf(r.s) < INFINITY;             // no NaN, no +infinity
        if (kOp == kListTop && first) {
            logp_row(a, row, live, r, zt);
            if (a.rank) a.rank[row] = good ? (int)before + 1 : 0;
        }
        if (!good) {
            no_list(live ? NAN : 0.f);
            if (kOp != kListTop && first) write_draw(a, row, -1, live ? NAN : 0.f, live ? NAN : 0.f, live ? NAN : 0.f);
        } else if constexpr (kAll) {
            if (warp == 0)
                draw_all<T>(a, row, r, IndexView<T>{z, a.V}, segment, uniform_of(a, random),
                            [&](int i) { return i >= rank * per && (C == 1 || i < (rank + 1) * per); }, lane);
        } else {
            if (n_keys > (uint32_t)sh.cap) {
                // ---- too many (the same in all CTAs of the row): a bound from all keys
                const uint64_t bound = bound_of_all<T, kThreads>(
                    view, v_lo, v_hi, (uint32_t)a.K, (uint32_t)sh.cap, own.hist, &pick, tid, [] { __syncthreads(); }, meet,
                    [&](const uint32_t* bin) {
                        if (C == 1) return *bin;
                        uint32_t n = 0;
                        for (int c = 0; c < C; ++c) n += peer_load(bin, c);
                        return n;
                    });
                meet();                                              // the counts that were read
                if (tid == 0) own.count = 0;
                __syncthreads();
                each_entry(view, v_lo, v_hi, tid, kThreads, [&](int j, float e) {
                    const uint64_t key = entry_key(e, j);
                    if (key >= bound) keys[atomicAdd(&own.count, 1u)] = key;
                });
                meet();
            }
            // ---- sorted in the first CTA
            int n = (int)own.count;
            if (C > 1 && rank == 0) {
                // CTA c's keys come after those of the ones before, by the warps w with w mod (C - 1) = c - 1
                const int mine = lane < C ? (int)peer_load(&own.count, lane) : 0;
                int upto = mine;
#pragma unroll
                for (int o = 1; o < 8; o *= 2) {
                    const int q = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += q;
                }
                const int c = 1 + warp % (C - 1), share = warp / (C - 1), shares = (kWarps - c) / (C - 1) + 1;
                const int more = __shfl_sync(0xffffffffu, mine, c), from = __shfl_sync(0xffffffffu, upto, c) - more;
                for (int i = 32 * share + lane; i < more; i += 32 * shares) keys[from + i] = peer_load(keys + i, c);
                n = __shfl_sync(0xffffffffu, upto, C - 1);
            }
            meet();                                                  // the other CTAs are done
            if (rank == 0) {
                const auto sort = [&] {
                    const Buckets b{order_key(r.m), own.hist, warp_total, order};
                    return sort_keys<kThreads>(keys, sorted, n, a.K, std::is_same<T, __nv_bfloat16>::value && a.V <= 65536, tid,
                                               [] { __syncthreads(); }, b);
                };
                const uint64_t* list = sort();
                // Slices that list a share of K each: all entries from `reach` on are there. Where the first K go
                // further down, this CTA finds them in the whole row.
                if (C > 1 && sh.slice_K < a.K && n_keys <= (uint32_t)sh.cap && reach > 0 &&
                    (n < a.K || (uint32_t)(list[a.K - 1] >> 40) < reach)) {
                    __syncthreads();
                    const auto sync = [] { __syncthreads(); };
                    const uint64_t bound = bound_of_all<T, kThreads>(view, 0, nv, (uint32_t)a.K, (uint32_t)sh.cap, own.hist, &pick, tid,
                                                                     sync, sync, [](const uint32_t* bin) { return *bin; });
                    if (tid == 0) n_again = 0;
                    __syncthreads();
                    each_entry(view, 0, nv, tid, kThreads, [&](int j, float e) {
                        const uint64_t key = entry_key(e, j);
                        if (key >= bound) keys[atomicAdd(&n_again, 1u)] = key;
                    });
                    __syncthreads();
                    n = (int)n_again;
                    list = sort();
                }
                if (kOp == kListDraw) {
                    if (warp == 0) draw_listed(a, row, r, list, min(n, a.K), lane);
                } else {
                    for (int i = tid; i < a.K; i += kThreads) {
                        const int64_t o = row * a.K + i;
                        a.top_ids[o] = i < n ? key_index(list[i]) : -1;
                        a.top_logp[o] = i < n ? log_prob(a, r, key_logit(list[i])) : -INFINITY;
                    }
                }
            }
        }
        // nothing of this row is read any more; of a list, nothing from peers since they met last
        if (kAll || !good) meet();
        else __syncthreads();
    }
    if (kAll && C > 1 && !met) cluster_wait();       // (no row was read)
}

template <class T, int kOp, int kThreads, int kMode>
cudaError_t launch_list_mode(const ListArgs& a, const ListShape& sh, size_t bytes, cudaStream_t s) {
    const auto kernel = token_list_kernel<T, kOp, kThreads, kMode>;
    if (bytes > 32 << 10) {                          // (one limit for all calls: threads may set it at once)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kListMost);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[2] = {};
    const int64_t rows = a.n < 1 << 20 ? a.n : 1 << 20;              // by a CTA or cluster each, the others by them too
    cfg.gridDim = dim3((unsigned)(rows * sh.cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits for the one before
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (sh.cluster > 1) {
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = sh.cluster;
        at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&cfg, kernel, a, sh);
}

template <class T, int kOp, int kThreads>
cudaError_t launch_list_threads(const ListArgs& a, ListShape sh, cudaStream_t s) {
    constexpr int kBatch = kThreads * kListPer;
    const int64_t batches = (sh.slice + kBatch - 1) / kBatch;
    int mode = batches > kManyBatches ? kLong : kCoarse;
    size_t bytes = (size_t)sh.cluster * batches * (kThreads / 32) * sizeof(float2);
    if (kOp != kListDrawAll) {
        // Maxima of as large groups as leave four for every entry of the list; none where the list takes a large
        // part of the slice.
        size_t maxima = 0;
        if (mode == kCoarse) mode = kEntries;
        if (sh.slice >= 2 * sh.slice_K) {
            if (mode == kEntries && 2 * sh.slice_K <= kThreads && sh.slice >= kBatch / 2) {
                mode = kCoarse;
                sh.group_log = 3;
                maxima = batches * kWords * kThreads * sizeof(uint32_t);
            } else if (kThreads >= 128 && mode == kEntries && 4 * (int64_t)sh.slice_K <= batches * kWords * kThreads) {
                mode = kWide;
                sh.group_log = 2;
                maxima = batches * kWords * kThreads * sizeof(uint32_t);
            } else {
                if (mode == kEntries) mode = kFine;
                sh.group_log = 0;
                while (sh.group_log < 2 && sh.slice >= (int64_t)sh.slice_K << (sh.group_log + 3)) ++sh.group_log;
                while (batches * kBatch >> sh.group_log > kListGroups) ++sh.group_log;
                maxima = ((batches * kListPer + (1 << sh.group_log) - 1) >> sh.group_log) * kThreads * sizeof(uint16_t);
            }
        }
        const int most = sh.slice_K * sh.cluster;
        sh.cap = sh.group_log < 0 || most > 256 ? kListCap : most > 64 ? 1024 : 512;
        sh.room = a.K <= 128 ? 128 : a.K <= 256 ? 256 : 1024;
        sh.maxima = (int)((maxima + 15) / 16 * 16);
        bytes = (size_t)(sh.cap + sh.room) * sizeof(uint64_t) + sh.maxima + sh.cap * sizeof(uint16_t);
    }
    if constexpr (kThreads > 128) {
        if (mode == kLong) return launch_list_mode<T, kOp, kThreads, kLong>(a, sh, bytes, s);
    }
    if constexpr (kOp != kListDrawAll) {
        if (mode == kFine) return launch_list_mode<T, kOp, kThreads, kFine>(a, sh, bytes, s);
        if constexpr (kThreads >= 128) {
            if (mode == kWide) return launch_list_mode<T, kOp, kThreads, kWide>(a, sh, bytes, s);
        }
        if (mode == kEntries) return launch_list_mode<T, kOp, kThreads, kEntries>(a, sh, bytes, s);
    }
    return launch_list_mode<T, kOp, kThreads, kCoarse>(a, sh, bytes, s);
}

}  // namespace

}  // namespace malib
