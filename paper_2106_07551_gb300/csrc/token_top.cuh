// A row's list of entries, by one warp: of the scores, the slopes at their log-probabilities; of
// distillation, the teacher's:
//   q_k = exp((t_k - max t) / T) / sum,  l = T^2 sum_k q_k (ln q_k - ln p_k).
// With ln p_k = (z_k - m) / T - ln S the student's part is sum_k q_k z_k / T alone; it is
// taken relative to the largest of the z_k, so that large logits lose nothing.
#pragma once

#include "token_emit.cuh"

namespace malib {

struct TopEntry {
    int id;                                          // -1: absent, < -1: counted at place -2 - id
    float q, z;                                      // the teacher's probability, or the slope; the student's logit
};
struct TopRow {
    float h;                                         // sum q ln q
    float zr, zq;                                    // a reference logit, sum q (z - zr) / T
    float q;                                         // sum q, over the entries with q != 0; or the slopes' sum
    int32_t live;                                    // the list has an entry
};

__device__ __forceinline__ float teacher_at(const TokenArgs& a, int64_t i) {
    if (a.tdtype == MALIB_F32) return static_cast<const float*>(a.teacher)[i];
    if (a.tdtype == MALIB_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(a.teacher)[i]);
    return __half2float(static_cast<const __half*>(a.teacher)[i]);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A row's entries with their logits at z (every lane of a warp): kScores, the ids with their slopes
// and the token with its own behind them; else the teacher's, of which logits of -infinity are absent.
// list has room for all of them. What an id that is listed more than once has goes to its first place
// later (id -2 - place): places are looked for where a bit of the id's low bits has been seen, 32
// entries at a time. Whether any is; and of the entries' slopes or teacher logits and of their
// logits the largest, by lane.
template <class T, int kBits, bool kScores>
__device__ __forceinline__ bool list_places(const TokenArgs& a, int64_t row, const T* z, int token, float slope,
                                            TopEntry* list, uint32_t (&seen)[kBits / 32], float& m, float& zr) {
    const int lane = threadIdx.x & 31, n = list_room(kScores ? kTokScoresList : kTokDistill, a.top);
    for (int i = lane; i < kBits / 32; i += 32) seen[i] = 0u;
    __syncwarp();
    m = zr = -INFINITY;
    bool twice = false;
    for (int j0 = 0; j0 < n; j0 += 32) {
        const int j = j0 + lane;
        int id = -1;
        float t = -INFINITY, zj = 0.f;
        if (j < a.top) {
            id = a.ids[row * a.top + j];
            t = kScores ? a.list_grad[row * a.top + j] : teacher_at(a, row * a.top + j);
            if (id >= a.V) {
                atomicOr(a.err, ERRBIT_BAD_TOKEN);
                id = -1;
            }
            if (id < 0 || (!kScores && t == -INFINITY)) id = -1;
        }
        if (kScores && j == a.top) {
            id = token;
            t = slope;
        }
        uint32_t* word = &seen[(id >> 5) & (kBits / 32 - 1)];
        const uint32_t bit = 1u << (id & 31);
        bool maybe = false;
        if (id >= 0) {
            m = max_nan(m, t);
            zj = Elt<T>::get(z[id]);
            zr = fmaxf(zr, zj);
            maybe = (*word & bit) != 0u;
        }
        __syncwarp();
        if (id >= 0) atomicOr(word, bit);
        int first = j;                               // the id's first place
        for (unsigned left = __ballot_sync(0xffffffffu, maybe); left; left &= left - 1) {
            const int u = __ffs(left) - 1, uid = __shfl_sync(0xffffffffu, id, u);
            for (int i0 = 0; i0 < j0; i0 += 32) {
                const unsigned hit = __ballot_sync(0xffffffffu, list[i0 + lane].id == uid);
                if (hit) {
                    if (lane == u) first = i0 + __ffs(hit) - 1;
                    break;
                }
            }
        }
        const int leader = __ffs(__match_any_sync(0xffffffffu, id)) - 1;
        first = __shfl_sync(0xffffffffu, first, leader);
        const bool later = id >= 0 && first != j;
        twice |= later;
        if (j < n) list[j] = TopEntry{later ? -2 - first : id, t, zj};
        __syncwarp();
    }
    return __any_sync(0xffffffffu, twice);
}
// Adds what entries have that were listed before, in the list's order (every lane of a warp). Only those are
// gone through: a row whose token is one of its listed entries has one, which is the usual case of scores.
// (Gradients of scores with the token among 64 entries, 4,096 x 32,768 bf16, 110 us with a walk through the
// whole list and 97 so, as without; among 1,024 1,074 and 593.)
__device__ __forceinline__ void join_places(TopEntry* list, int n, bool twice) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
    for (int j0 = 0; twice && j0 < n; j0 += 32) {
        const bool more = j0 + lane < n && list[j0 + lane].id < -1;
        for (unsigned left = __ballot_sync(0xffffffffu, more); left; left &= left - 1) {
            const TopEntry& e = list[j0 + __ffs(left) - 1];
            if (lane == 0) list[-2 - e.id].q += e.q;
        }
    }
    __syncwarp();
}

// The list of a row whose logits are at z (every lane of a warp); list has room for
// a.top entries.
template <class T, int kBits>
__device__ __forceinline__ TopRow top_row(const TokenArgs& a, int64_t row, const T* z, TopEntry* list,
                                          uint32_t (&seen)[kBits / 32]) {
    const int lane = threadIdx.x & 31;
    float m, zr;
    const bool twice = list_places<T, kBits, false>(a, row, z, -1, 0.f, list, seen, m, zr);
    m = warp_max_nan(m);
    zr = warp_max_nan(zr);
    if (!(fabsf(zr) < INFINITY)) zr = 0.f;
    float s = 0.f;
    for (int j = lane; j < a.top; j += 32)
        if (list[j].id != -1) s += expf((list[j].q - m) * a.inv_t);
    const float ls = logf(warp_sum(s));
    float h = 0.f, zq = 0.f, qs = 0.f;
    for (int j = lane; j < a.top; j += 32) {
        const TopEntry e = list[j];
        if (e.id == -1) continue;
        const float lq = (e.q - m) * a.inv_t - ls, q = expf(lq);
        list[j].q = q;
        if (q != 0.f) {
            h = fmaf(q, lq, h);
            zq = fmaf(q, (e.z - zr) * a.inv_t, zq);
            qs += q;
        }
    }
    join_places(list, a.top, twice);
    return TopRow{warp_sum(h), zr, warp_sum(zq), warp_sum(qs), m != -INFINITY};
}

// The slopes of a row at its token's and the listed entries' log-probabilities, each entry once;
// their sum in q (every lane of a warp). list has room for a.top + 1 entries.
template <class T, int kBits>
__device__ __forceinline__ TopRow scores_list(const TokenArgs& a, int64_t row, const T* z, int token, TopEntry* list,
                                              uint32_t (&seen)[kBits / 32]) {
    const int lane = threadIdx.x & 31;
    float m, zr, sum = 0.f;
    const float slope = a.logp_grad ? a.logp_grad[row] : 0.f;
    const bool twice = list_places<T, kBits, true>(a, row, z, token, slope, list, seen, m, zr);
    for (int j = lane; j <= a.top; j += 32)
        if (list[j].id != -1) sum += list[j].q;
    join_places(list, a.top + 1, twice);
    return TopRow{0.f, 0.f, 0.f, warp_sum(sum), 1};
}
// What the list kOp takes of a row.
template <class T, int kOp, int kBits>
__device__ __forceinline__ TopRow list_row(const TokenArgs& a, int64_t row, const T* z, int token, TopEntry* list,
                                           uint32_t (&seen)[kBits / 32]) {
    if constexpr (kOp == kTokScoresList) return scores_list<T, kBits>(a, row, z, token, list, seen);
    else return top_row<T, kBits>(a, row, z, list, seen);
}
// The gradient at an entry of the list.
template <int kOp>
__device__ __forceinline__ float list_entry(const TopEntry& e, const RowGrad& c, float k) {
    const float x = x_of(e.z, c.m, k), p = exp2_fast(x);
    if (kOp == kTokDistill) return c.c0 * p - c.at * e.q;
    return emit_steep(e.z, RowGrad{c.m, c.c0, c.c1, c.at * e.q}, k, true);
}

// The row's loss.
__device__ __forceinline__ float top_loss(const TokenArgs& a, const RowStat& r, const TopRow& t) {
    // sum q ln p = sum q (z - zr) / T + ((zr - m) / T - ln S) sum q
    const float lp = fmaf(log_prob(a, r, t.zr), t.q, t.zq);
    return a.tt * (t.h - lp);
}

}  // namespace malib
