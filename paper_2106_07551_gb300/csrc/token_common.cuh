// Losses of token policies: what the kernels share. A row holds the logits z_0 ..
// z_{V-1} of one position; with a temperature T, y = z / T,
//   p_j = exp(y_j - max y) / S,  S = sum_j exp(y_j - max y),
//   ln p_j = y_j - max y - ln S,  H = ln S - (1 / S) sum_j exp(y_j - max y) (y_j - max y).
// Everything is computed in base 2 on x_j = (z_j - m) k, m = max z, k = log2(e) / T:
// p_j = 2^x_j / S. The difference is taken before the product, so that neither the
// lowest finite values of a type nor large logits overflow on the way, and a row of
// equal values of any size is uniform.
// A row's statistics are (m, S, t), t = sum_j 2^x_j x_j, gathered in one pass over the
// row with a running maximum; two partial statistics combine by scaling with
// 2^((m_a - m) k). They are held in fp32: a row's sum has at most a few hundred
// thousand terms, added in thousands of partial sums.
// x is held above -200, where 2^x is 0 in fp32, wherever it multiplies 2^x: an entry
// of -infinity (masked) contributes 0 and not 0 x infinity. A NaN or +infinity makes
// the row's S, and with it all that follows from the row, NaN.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "device_common.cuh"

namespace malib {

constexpr int kTokenMaxTop = 1024;                   // teacher entries of a row
constexpr int kTokenStats = 5;                       // sums of a call's statistics
constexpr int kTokenMaxCtas = 8192;                  // CTAs whose partial sums the work space holds

enum : int { kTokLogp = 0, kTokPpo = 1, kTokDistill = 2 };

// What a row's statistics leave for a preference pair's sums and its gradient.
struct TokenRow {
    float m, inv_s, logp;
    int32_t live;
};

struct TokenArgs {
    const void* z;               // [n][ld]
    int64_t ld;
    void* g;                     // [n][gld], the gradient; null: none
    int64_t gld;
    int64_t n;
    int32_t V;
    int32_t dtype;
    float k, inv_t;              // log2(e) / T, 1 / T
    const int32_t* tokens;       // [n], < 0: the row is left out
    int* err;
    // policy loss, distillation
    const float* weight;         // [n]; null: w0
    float w0;
    float gscale;                // gradients are multiplied by it
    const float* old_logp;
    const float* adv;
    const float* ref;            // null: no KL term
    float ratio_lo, ratio_hi;    // clip range of the ratio
    float kl, ent;
    // distillation
    const int32_t* ids;          // [n][top], < 0: absent
    const void* teacher;         // [n][top]
    int32_t tdtype, top;
    float tt;                    // T^2
    // preference pairs
    const int64_t* offsets;      // [2 pairs + 1]
    int32_t n_pairs;
    float beta, smooth;
    float* pair_coef;            // [n_pairs] d loss / d (reward difference), scaled for the gradient
    TokenRow* rows;              // [n]
    // results
    float* logp;
    float* entropy;
    float* loss;
    float* reward;               // [2 n_pairs]
    float* stats;
    double* part;                // [kTokenMaxCtas][kTokenStats]
    unsigned* ticket;            // CTAs that have written their partial sums
};

template <class T>
struct Elt;                      // W elements in 16 bytes
template <>
struct Elt<float> {
    static constexpr int W = 4;
    __device__ static float get(float v) { return v; }
    __device__ static float put(float v) { return v; }
    __device__ static void unpack(const uint4& q, float (&v)[4]) {
        v[0] = __uint_as_float(q.x);
        v[1] = __uint_as_float(q.y);
        v[2] = __uint_as_float(q.z);
        v[3] = __uint_as_float(q.w);
    }
    __device__ static uint4 pack(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <>
struct Elt<__nv_bfloat16> {
    static constexpr int W = 8;
    __device__ static float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ static __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
    __device__ static void unpack(const uint4& q, float (&v)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static uint4 pack(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Elt<__half> {
    static constexpr int W = 8;
    __device__ static float get(__half v) { return __half2float(v); }
    __device__ static __half put(float v) { return __float2half_rn(v); }
    __device__ static void unpack(const uint4& q, float (&v)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __half2 h;
            *reinterpret_cast<uint32_t*>(&h) = w[i];
            const float2 f = __half22float2(h);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
    __device__ static uint4 pack(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kXMin = -200.f;

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

struct RowStat {
    float m, s, t;
};

// b's sums join a's. A side that has seen only -infinity has s = t = 0.
__device__ __forceinline__ RowStat combine(const RowStat& a, const RowStat& b, float k) {
    RowStat r;
    r.m = max_nan(a.m, b.m);
    // (-infinity) - (-infinity) is NaN, which fmaxf takes for kXMin: a factor 0 on sums of 0
    const float da = fmaxf((a.m - r.m) * k, kXMin), db = fmaxf((b.m - r.m) * k, kXMin);
    const float fa = exp2_fast(da), fb = exp2_fast(db);
    r.s = fmaf(a.s, fa, b.s * fb);
    r.t = fa * fmaf(a.s, da, a.t) + fb * fmaf(b.s, db, b.t);
    return r;
}

// W further entries of a row join r.
template <int W>
__device__ __forceinline__ void add_entries(RowStat& r, const float (&v)[W], float k) {
    float mx = v[0];
#pragma unroll
    for (int i = 1; i < W; ++i) mx = max_nan(mx, v[i]);
    if (!(mx <= r.m)) {                              // a new maximum, or a NaN
        const float m = max_nan(r.m, mx);
        const float d = fmaxf((r.m - m) * k, kXMin), f = exp2_fast(d);
        r.t = f * fmaf(r.s, d, r.t);
        r.s *= f;
        r.m = m;
    }
    if (r.m == -INFINITY) return;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float x = (v[i] - r.m) * k;
        const float e = exp2_fast(x);
        r.s += e;
        r.t = fmaf(e, fmaxf(x, kXMin), r.t);
    }
}

// Statistics of the whole block, the same in every thread. red: a slot a warp.
template <int kWarps>
__device__ __forceinline__ RowStat block_stat(RowStat r, float k, RowStat* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        RowStat b;
        b.m = __shfl_xor_sync(0xffffffffu, r.m, o);
        b.s = __shfl_xor_sync(0xffffffffu, r.s, o);
        b.t = __shfl_xor_sync(0xffffffffu, r.t, o);
        r = combine(r, b, k);
    }
    if (lane == 0) red[warp] = r;
    __syncthreads();
    r = red[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) r = combine(r, red[w], k);
    return r;
}

// The gradient at entry j is 2^x_j (c0 + c1 x_j), and `at` more at the row's token.
struct RowGrad {
    float m, c0, c1, at;
};

// ln p of the entry with logit z.
__device__ __forceinline__ float log_prob(const RowStat& r, float z, float inv_t) {
    return (z - r.m) * inv_t - logf(r.s);
}
__device__ __forceinline__ float row_entropy(const RowStat& r) {
    return logf(r.s) - kLn2 * (r.t / r.s);
}

// The clipped policy loss of one row (l, before its weight) and its gradient.
__device__ __forceinline__ RowGrad ppo_row(const TokenArgs& a, int64_t row, const RowStat& r, float logp, float w,
                                           float* loss, float* clipped, float* kl, float* H) {
    const float A = a.adv[row];
    const float rho = expf(logp - a.old_logp[row]);
    const float free_ = rho * A;
    // a NaN ratio stays one (fminf and fmaxf would drop it)
    const float cut = (rho < a.ratio_lo ? a.ratio_lo : rho > a.ratio_hi ? a.ratio_hi : rho) * A;
    const bool clip = free_ > cut;                   // ties to the unclipped term, which carries the gradient
    *H = row_entropy(r);
    float l = -(clip ? cut : free_) - a.ent * *H;
    float slope = clip ? 0.f : -free_;               // d l / d ln p of the token
    *kl = 0.f;
    if (a.ref) {
        const float d = a.ref[row] - logp, e = expm1f(d);
        *kl = e - d;
        l = fmaf(a.kl, *kl, l);
        slope = fmaf(-a.kl, e, slope);
    }
    *loss = l;
    *clipped = clip ? 1.f : 0.f;
    const float f = w * a.gscale * a.inv_t;
    const float gt = f * slope, h = f * a.ent, inv_s = 1.f / r.s;
    // p (-gt + h (ln p + H)),  ln p = x ln 2 - ln S
    return RowGrad{r.m, inv_s * (a.ent != 0.f ? fmaf(h, *H - logf(r.s), -gt) : -gt), inv_s * h * kLn2, gt};
}

// Partial sums of a call's statistics: the CTA's, then, in the CTA that comes last,
// the call's, in a fixed order. Returns in thread 0 of that CTA true with the sums in
// out. Called by every thread of the block; acc is thread 0's.
template <int kThreads>
__device__ __forceinline__ bool sum_partials(double* part, unsigned* ticket, const double (&acc)[kTokenStats],
                                             double (&out)[kTokenStats]) {
    __shared__ bool last;
    __shared__ double red[kThreads / 32][kTokenStats];
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 0; i < kTokenStats; ++i) part[(int64_t)blockIdx.x * kTokenStats + i] = acc[i];
        __threadfence();
        last = atomicInc(ticket, gridDim.x - 1) == gridDim.x - 1;   // back at 0 for the next call
    }
    __syncthreads();
    if (!last) return false;
    __threadfence();
    double v[kTokenStats] = {};
    for (int c = threadIdx.x; c < (int)gridDim.x; c += kThreads)
#pragma unroll
        for (int i = 0; i < kTokenStats; ++i) v[i] += __ldcg(part + (int64_t)c * kTokenStats + i);
#pragma unroll
    for (int i = 0; i < kTokenStats; ++i) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5][i] = v[i];
    }
    __syncthreads();
    if (threadIdx.x != 0) return false;
#pragma unroll
    for (int i = 0; i < kTokenStats; ++i) {
        out[i] = 0.0;
        for (int w = 0; w < kThreads / 32; ++w) out[i] += red[w][i];
    }
    return true;
}

cudaError_t launch_token_rows(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_pairs(const TokenArgs& a, int n_sm, cudaStream_t s);

}  // namespace malib
