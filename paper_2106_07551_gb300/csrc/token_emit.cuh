// Losses of token policies: a part of a row's gradient from its logits in shared memory.
#pragma once

#include "token_common.cuh"
#include "token_shift.cuh"

namespace malib {

namespace {

// One entry of the gradient.
template <class T>
__device__ __forceinline__ float emit_one(T z, const RowGrad& c, float k) {
    const float x = x_of(Elt<T>::get(z), c.m, k);
    return exp2_fast(x) * fmaf(c.c1, fmaxf(x, kXMin), c.c0);
}

// A row of the policy loss whose slope at ln p is infinite (a KL term or a ratio past fp32, a
// masked token with a KL term): its entries are infinite, and 0 times infinity or the difference
// of two infinities would make NaN of some. One entry of such a row, or of any other: 0 where p is
// 0, the slope's sign at the token.
__device__ __forceinline__ bool is_steep(const RowGrad& c) { return fabsf(c.c0) == INFINITY; }
template <class T>
__device__ __forceinline__ float emit_steep(T z, const RowGrad& c, float k, bool token) {
    const float x = x_of(Elt<T>::get(z), c.m, k), e = exp2_fast(x);
    const float v = e == 0.f && is_steep(c) ? 0.f : e * fmaf(c.c1, fmaxf(x, kXMin), c.c0);
    return !token ? v : fabsf(c.at) == INFINITY ? c.at : v + c.at;
}
// Sixteen bytes of such a row, the token entry `at` of them.
template <class T>
__device__ __forceinline__ void emit_steep(const uint4& q, const RowGrad& c, float k, int at, F2 (&v)[Elt<T>::W / 2]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < Elt<T>::W; i += 2)
        v[i / 2] = f2_make(emit_steep(Elt<T>::word(w, i), c, k, i == at), emit_steep(Elt<T>::word(w, i + 1), c, k, i + 1 == at));
}
// Entries [j0, j1), entry j at e[j], by kThreads threads tid.
template <class T, int kThreads>
__device__ __forceinline__ void emit_steep_part(int tid, const T* e, int j0, int j1, T* g, const RowGrad& c, float k,
                                                int token) {
#pragma unroll 1
    for (int j = j0 + tid; j < j1; j += kThreads) g[j] = Elt<T>::put(emit_steep(e[j], c, k, j == token));
}

// The gradient of a stage: entries [j0, j1) of the row, those of the n vectors at src,
// the first of which is entry `first` (before the row where the row starts inside it). By
// the first kConsumers threads; a full stage has kPer vectors for each.
template <class T, bool kEntropy, int kConsumers, int kPer>
__device__ __forceinline__ void emit_stage(int tid, const uint8_t* src, int first, int j0, int j1, int n, T* g, bool alike,
                                           const RowGrad& c, float k, int token) {
    constexpr int W = Elt<T>::W;
    const T* e = reinterpret_cast<const T*>(src) - first;            // entry j at e[j]
    F2 v[W / 2];
    if (alike) {
        const uint4* q = reinterpret_cast<const uint4*>(src) + tid;
        T* out = g + (first + tid * W);
        if (j0 == first && j1 - j0 == kPer * kConsumers * W) {
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                emit<T, kEntropy>(q[u * kConsumers], c, k, v);
                __stcs(reinterpret_cast<uint4*>(out + u * kConsumers * W), Elt<T>::pack(v));
            }
        } else {
            for (int i = tid; i < n; i += kConsumers, q += kConsumers, out += kConsumers * W) {
                emit<T, kEntropy>(*q, c, k, v);
                const int j = first + i * W;
                if (j >= j0 && j + W <= j1) __stcs(reinterpret_cast<uint4*>(out), Elt<T>::pack(v));
                else store_part(out, j - j0, j1 - j0, Elt<T>::pack(v));
            }
        }
        // the token's entry, by the thread that has just written it
        if (token >= j0 && token < j1 && (token - first) / W % kConsumers == tid)
            g[token] = Elt<T>::put(emit_one(e[token], c, k) + c.at);
    } else {
        // vectors of the gradient's own alignment, entry by entry what is left at the ends
        const int to = (int)((16u - ((uintptr_t)(g + j0) & 15u) & 15u) / sizeof(T));
        const int a0 = min(j0 + to, j1), nv = (j1 - a0) / W, a1 = a0 + nv * W;
        const uint8_t* p = reinterpret_cast<const uint8_t*>(e + a0);
        const int by = (int)((uintptr_t)p & 15u);
        p -= by;
        for (int i = tid; i < nv; i += kConsumers) {
            emit<T, kEntropy>(load_shifted(p + i * 16, by), c, k, v);
            __stcs(reinterpret_cast<uint4*>(g + (a0 + i * W)), Elt<T>::pack(v));
        }
        const int j = tid < W ? j0 + tid : a1 + tid - W;
        if (tid < 2 * W && j < (tid < W ? a0 : j1)) g[j] = Elt<T>::put(emit_one(e[j], c, k));
        if (token >= j0 && token < j1) {
            const int owner = token < a0 ? token - j0 : token >= a1 ? token - a1 + W : (token - a0) / W % kConsumers;
            if (owner == tid) g[token] = Elt<T>::put(emit_one(e[token], c, k) + c.at);
        }
    }
}

// Zeros to entries [j0, j1) of a row, by kConsumers threads tid.
template <class T, int kConsumers>
__device__ __forceinline__ void zero_entries(int tid, T* g, int j0, int j1) {
    constexpr int W = Elt<T>::W;
    const int to = (int)((16u - ((uintptr_t)(g + j0) & 15u) & 15u) / sizeof(T));
    const int a0 = min(j0 + to, j1), nv = (j1 - a0) / W, a1 = a0 + nv * W;
    for (int i = tid; i < nv; i += kConsumers)
        __stcs(reinterpret_cast<uint4*>(g + (a0 + i * W)), make_uint4(0, 0, 0, 0));
    const int j = tid < W ? j0 + tid : a1 + tid - W;
    if (tid < 2 * W && j < (tid < W ? a0 : j1)) g[j] = Elt<T>::put(0.f);
}

}  // namespace

}  // namespace malib
