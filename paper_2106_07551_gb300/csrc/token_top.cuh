// Distillation: a row's list of teacher entries, by one warp.
//   q_k = exp((t_k - max t) / T) / sum,  l = T^2 sum_k q_k (ln q_k - ln p_k).
// With ln p_k = (z_k - m) / T - ln S the student's part is sum_k q_k z_k / T alone; it is
// taken relative to the largest of the z_k, so that large logits lose nothing.
#pragma once

#include "token_common.cuh"

namespace malib {

struct TopEntry {
    int id;                                          // -1: absent, < -1: counted at place -2 - id
    float q, z;                                      // the teacher's probability, the student's logit
};
struct TopRow {
    float h;                                         // sum q ln q
    float zr, zq;                                    // a reference logit, sum q (z - zr) / T
    float q;                                         // sum q, over the entries with q != 0
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

// The list of a row whose logits are at z (every lane of a warp); list has room for
// a.top entries. Teacher logits of -infinity are absent. The q of an id that is listed
// more than once are added, in the list's order, at its first place: places are looked
// for where a bit of the id's low bits has been seen, 32 entries at a time.
template <class T, int kBits>
__device__ __forceinline__ TopRow top_row(const TokenArgs& a, int64_t row, const T* z, TopEntry* list,
                                          uint32_t (&seen)[kBits / 32]) {
    const int lane = threadIdx.x & 31;
    for (int i = lane; i < kBits / 32; i += 32) seen[i] = 0u;
    __syncwarp();
    float m = -INFINITY, zr = -INFINITY;
    bool twice = false;
    for (int j0 = 0; j0 < a.top; j0 += 32) {
        const int j = j0 + lane;
        int id = -1;
        float t = -INFINITY, zj = 0.f;
        if (j < a.top) {
            id = a.ids[row * a.top + j];
            t = teacher_at(a, row * a.top + j);
            if (id >= a.V) {
                atomicOr(a.err, ERRBIT_BAD_TOKEN);
                id = -1;
            }
            if (id < 0 || t == -INFINITY) id = -1;
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
        if (j < a.top) list[j] = TopEntry{later ? -2 - first : id, t, zj};
        __syncwarp();
    }
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
    __syncwarp();
    if (__any_sync(0xffffffffu, twice) && lane == 0)
        for (int j = 0; j < a.top; ++j)
            if (list[j].id < -1) list[-2 - list[j].id].q += list[j].q;
    __syncwarp();
    return TopRow{warp_sum(h), zr, warp_sum(zq), warp_sum(qs), m != -INFINITY};
}

// The row's loss.
__device__ __forceinline__ float top_loss(const TokenArgs& a, const RowStat& r, const TopRow& t) {
    // sum q ln p = sum q (z - zr) / T + ((zr - m) / T - ln S) sum q
    const float lp = fmaf(log_prob(a, r, t.zr), t.q, t.zq);
    return a.tt * (t.h - lp);
}

}  // namespace malib
