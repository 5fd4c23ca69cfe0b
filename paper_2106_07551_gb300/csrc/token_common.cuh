// Losses of token policies: what the kernels share. A row holds the logits z_0 ..
// z_{V-1} of one position; with a temperature T, y = z / T,
//   p_j = exp(y_j - max y) / S,  S = sum_j exp(y_j - max y),
//   ln p_j = y_j - max y - ln S,  H = ln S - (1 / S) sum_j exp(y_j - max y) (y_j - max y).
// Everything is computed in base 2 on x_j = (z_j - m) k, m = max z, k = log2(e) / T:
// p_j = 2^x_j / S. The difference is taken before the product, so that neither the
// lowest finite values of a type nor large logits overflow on the way, a row of equal
// values of any size is uniform, and S >= 1: no ln p is above 0. (One fused
// multiply-add z k - m k would save an operation for fp32 logits; 16-bit ones are
// widened by the subtraction itself.)
// A row's statistics are (m, S, t), t = sum_j 2^x_j x_j, gathered in one pass over the
// row with a running maximum; two partial statistics combine by scaling with
// 2^((m_a - m) k). They are held in fp32, a long row's with what the additions of its
// parts' sums leave (LongStat).
// The fast base-2 exponential is low by 5.0e-8 of its value on average (measured over
// [-20, 0), the same from -1 down), which every sum of a row, and every scaling of one,
// would pass on and a sequence's sum add up; 2^x is taken of x + kExpBias, added in the
// same rounding, which leaves 2^0 = 1.
// x is held above -200, where 2^x is 0 in fp32, wherever it multiplies 2^x: an entry
// of -infinity (masked) contributes 0 and not 0 x infinity. A NaN or +infinity makes
// the row's S, and with it all that follows from the row, NaN.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "device_common.cuh"
#include "f32x2.cuh"

namespace malib {

constexpr int kTokenMaxTop = 1024;                   // teacher entries of a row
constexpr int kTokenMaxCtas = 8192;                  // CTAs whose partial sums the work space holds

enum : int { kTokLogp = 0, kTokPpo = 1, kTokDistill = 2, kTokPairGrad = 3, kTokScores = 4, kTokScoresList = 5 };
// Calls whose gradient has a factor of ln p (and not of p alone), and one that may be infinite;
// calls that read a list of entries for every row; calls with statistics over the rows.
__host__ __device__ constexpr bool has_slope(int op) { return op == kTokPpo || op == kTokScores || op == kTokScoresList; }
__host__ __device__ constexpr bool has_list(int op) { return op == kTokDistill || op == kTokScoresList; }
__host__ __device__ constexpr bool has_stats(int op) { return op == kTokPpo || op == kTokDistill; }
// Entries that a row's list takes: the scores' one has the token behind the `top` given ones.
__host__ __device__ constexpr int list_room(int op, int top) { return op == kTokDistill ? top : op == kTokScoresList ? top + 1 : 0; }

// What a row's statistics leave for a preference pair's sums and its gradient: first
// value + rest is ln p of the token; the pair's sums put d L / d logit of the token
// before -p into value. inv_s = 0: the row is left out.
struct __align__(16) TokenRow {
    float m, inv_s, value, rest;
};

// A row's share of a call's statistics.
struct __align__(16) RowSum {
    float loss, x, y;                                // w l; policy loss: KL, H; distillation: l
    int32_t flags;                                   // bit 0: counted; bit 1: clipped
};

struct TokenArgs {
    const void* z;               // [n][ld]
    int64_t ld;
    void* g;                     // [n][gld], the gradient; null: none
    int64_t gld;
    int64_t n;
    int32_t V;
    int32_t dtype;
    float k, inv_t, inv_t_lo;    // log2(e) / T, 1 / T and what its rounding leaves
    float dk;                    // ln 2 times the relative error of k's rounding
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
    float tt, top_scale;         // T^2, T
    // scores: the loss's slopes
    const float* logp_grad;      // [n] at ln p of the row's token; null: 0
    const float* entropy_grad;   // [n] at H; null: 0
    const float* list_grad;      // [n][top] at ln p of the entries ids
    // preference pairs
    const int64_t* offsets;      // [2 pairs + 1]
    int32_t n_pairs;
    float beta, smooth;
    TokenRow* rows;              // [n]
    // results
    float* logp;
    float* entropy;
    float* loss;
    float* reward;               // [2 n_pairs]
    float* stats;
    struct Totals* part;         // [kTokenMaxCtas]
    unsigned* ticket;            // CTAs that have written their sums
    RowSum* row_sums;            // [n]
    unsigned long long* claims;  // rows claimed
};

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

using F2 = unsigned long long;                       // two floats
__device__ __forceinline__ F2 f2_make(float lo, float hi) {
    return f2_pack(__float_as_uint(lo), __float_as_uint(hi));
}
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <class T>
struct Elt;                      // W elements in 16 bytes
template <>
struct Elt<float> {
    static constexpr int W = 4;
    __device__ static uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }   // -infinity
    __device__ static float word(const uint32_t (&w)[4], int i) { return __uint_as_float(w[i]); }   // entry i
    __device__ static float get(float v) { return v; }
    __device__ static float put(float v) { return v; }
    // the entries, two by two
    __device__ static void pairs(const uint4& q, F2 (&v)[2]) {
        v[0] = f2_pack(q.x, q.y);
        v[1] = f2_pack(q.z, q.w);
    }
    // the maximum of two words' entries, NaN if one is NaN; and the largest entry of a word
    __device__ static uint32_t max(uint32_t a, uint32_t b) {
        return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    }
    __device__ static float largest(uint32_t m) { return __uint_as_float(m); }
    __device__ static uint4 pack(const F2 (&v)[2]) {
        const float2 a = f2_split(v[0]), b = f2_split(v[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
};
template <>
struct Elt<__nv_bfloat16> {
    static constexpr int W = 8;
    __device__ static uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }   // -infinity
    __device__ static __nv_bfloat16 word(const uint32_t (&w)[4], int i) {
        return __ushort_as_bfloat16((unsigned short)(w[i >> 1] >> 16 * (i & 1)));
    }
    __device__ static float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ static __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
    __device__ static void pairs(const uint4& q, F2 (&v)[4]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f2_pack(w[i] << 16, w[i] & 0xffff0000u);
    }
    __device__ static uint32_t max(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static float largest(uint32_t m) {
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    __device__ static uint4 pack(const F2 (&v)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = f2_split(v[i]);
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f.y), "f"(f.x));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Elt<__half> {
    static constexpr int W = 8;
    __device__ static uint4 none() { return make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u); }   // -infinity
    __device__ static __half word(const uint32_t (&w)[4], int i) {
        return __ushort_as_half((unsigned short)(w[i >> 1] >> 16 * (i & 1)));
    }
    __device__ static float get(__half v) { return __half2float(v); }
    __device__ static __half put(float v) { return __float2half_rn(v); }
    __device__ static void pairs(const uint4& q, F2 (&v)[4]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __half2 h;
            *reinterpret_cast<uint32_t*>(&h) = w[i];
            const float2 f = __half22float2(h);
            v[i] = f2_make(f.x, f.y);
        }
    }
    __device__ static uint32_t max(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static float largest(uint32_t m) {
        __half2 h;
        *reinterpret_cast<uint32_t*>(&h) = m;
        const float2 f = __half22float2(h);
        return max_nan(f.x, f.y);
    }
    __device__ static uint4 pack(const F2 (&v)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = f2_split(v[i]);
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f.y), "f"(f.x));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kXMin = -200.f;
constexpr float kExpBias = 7.3e-8f;                  // 5.04e-8 / ln 2

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ F2 f2_fma3(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ F2 f2_exp2(F2 x) {
    const float2 v = f2_split(x);
    return f2_make(exp2_fast(v.x), exp2_fast(v.y));
}
__device__ __forceinline__ F2 f2_floor_x(F2 x) {
    const float2 v = f2_split(x);
    return f2_make(fmaxf(v.x, kXMin), fmaxf(v.y, kXMin));
}

// A sum in fp32 with the rounding errors of its additions beside it (Knuth's two-sum): as
// good as one in fp64, whose rate is a sixtieth of fp32's here, over some 10^5 additions. The
// errors' own sum is plain fp32: it is off by 1e-6 to 4e-6 of the whole after 262,144 additions of
// one value, 1e-4 after 1.8 million. Where there may be as many it is settled as it goes, which
// keeps the errors' sum below half a unit of the whole.
struct Sum2 {
    float s, e;
    __device__ __forceinline__ void add(float x) {
        const float t = __fadd_rn(s, x), y = __fsub_rn(t, s);
        e = __fadd_rn(e, __fadd_rn(__fsub_rn(s, __fsub_rn(t, y)), __fsub_rn(x, y)));
        s = t;
    }
    __device__ __forceinline__ void add(const Sum2& b) {
        add(b.s);
        e = __fadd_rn(e, b.e);
    }
    // an infinite sum has an error that is NaN, and none to speak of
    __device__ __forceinline__ void settle() {
        if (!(fabsf(s) < INFINITY)) return;
        const float t = __fadd_rn(s, e);
        e = __fsub_rn(e, __fsub_rn(t, s));
        s = t;
    }
    __device__ __forceinline__ float value() const { return fabsf(s) < INFINITY ? __fadd_rn(s, e) : s; }
};
struct RowStat {
    float m, s, t;
};

// x of an entry with logit z in a row of maximum m, as 2^x takes it.
__device__ __forceinline__ float x_of(float z, float m, float k) { return fmaf(z - m, k, kExpBias); }

// b's sums join a's. A side that has seen only -infinity has s = t = 0.
__device__ __forceinline__ RowStat combine(const RowStat& a, const RowStat& b, float k) {
    RowStat r;
    r.m = max_nan(a.m, b.m);
    // (-infinity) - (-infinity) is NaN, which fmaxf takes for kXMin: a factor 0 on sums of 0
    const float da = fmaxf((a.m - r.m) * k, kXMin), db = fmaxf((b.m - r.m) * k, kXMin);
    const float fa = exp2_fast(da + kExpBias), fb = exp2_fast(db + kExpBias);
    r.s = fmaf(a.s, fa, b.s * fb);
    r.t = fa * fmaf(a.s, da, a.t) + fb * fmaf(b.s, db, b.t);
    return r;
}

// A running maximum takes in mx: sums so far are scaled to the new one.
__device__ __forceinline__ void raise(RowStat& r, float mx, float k) {
    if (mx <= r.m) return;                           // neither a new maximum nor a NaN
    const float m = max_nan(r.m, mx);
    const float d = fmaxf((r.m - m) * k, kXMin), f = exp2_fast(d + kExpBias);
    r.t = f * fmaf(r.s, d, r.t);
    r.s *= f;
    r.m = m;
}

// The maximum of 16-byte vectors of logits (NaN if one is NaN).
template <class T, int N>
__device__ __forceinline__ float vec_max(const uint4 (&q)[N]) {
    uint32_t m = q[0].x;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        if (u > 0) m = Elt<T>::max(m, q[u].x);
        m = Elt<T>::max(m, q[u].y);
        m = Elt<T>::max(m, q[u].z);
        m = Elt<T>::max(m, q[u].w);
    }
    return Elt<T>::largest(m);
}

// Vectors of logits join r, whose maximum covers them already and is not -infinity.
template <class T, int N>
__device__ __forceinline__ void gather(RowStat& r, const uint4 (&q)[N], float k) {
    constexpr int P = Elt<T>::W / 2;
    F2 s = 0ull, t = 0ull;
    const F2 k2 = f2_dup(k), neg = f2_dup(-r.m), bias = f2_dup(kExpBias);
#pragma unroll
    for (int u = 0; u < N; ++u) {
        F2 y[P];
        Elt<T>::pairs(q[u], y);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const F2 x = f2_fma3(f2_add(y[i], neg), k2, bias), e = f2_exp2(x);
            s = f2_add(s, e);
            f2_fma(t, e, f2_floor_x(x));
        }
    }
    const float2 s2 = f2_split(s), t2 = f2_split(t);
    r.s += s2.x + s2.y;
    r.t += t2.x + t2.y;
}

// The statistics of a row of many parts: each part's sums join these with the rounding errors of
// the additions kept, so that what a row of any length loses is what a part does. (One sum over
// 2^24 entries, 131,072 a thread, is off by up to 7e-4 of itself.)
struct LongStat {
    float m;
    Sum2 s, t;
};
__device__ __forceinline__ void raise(LongStat& r, float mx, float k) {
    if (mx <= r.m) return;
    const float m = max_nan(r.m, mx);
    const float d = fmaxf((r.m - m) * k, kXMin), f = exp2_fast(d + kExpBias);
    r.t = Sum2{f * fmaf(r.s.s, d, r.t.s), f * fmaf(r.s.e, d, r.t.e)};
    r.s = Sum2{f * r.s.s, f * r.s.e};
    r.m = m;
}
template <class T, int N>
__device__ __forceinline__ void gather(LongStat& r, const uint4 (&q)[N], float k) {
    RowStat part{r.m, 0.f, 0.f};
    gather<T>(part, q, k);
    r.s.add(part.s);
    r.t.add(part.t);
}
__device__ __forceinline__ RowStat stat_of(const LongStat& r) { return RowStat{r.m, r.s.value(), r.t.value()}; }
__device__ __forceinline__ RowStat stat_of(const RowStat& r) { return r; }

// Statistics of N lanes that follow one another, the same in each: their maximum, then
// their sums to its base.
template <int N>
__device__ __forceinline__ RowStat reduce_stat(RowStat r, float k) {
    float m = r.m;
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    r = combine(r, RowStat{m, 0.f, 0.f}, k);
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) {
        r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
        r.t += __shfl_xor_sync(0xffffffffu, r.t, o);
    }
    return r;
}

// The gradient at entry j is 2^x_j (c0 + c1 x_j), and `at` more at the row's token.
struct RowGrad {
    float m, c0, c1, at;
};

// The mean of x under p.
__device__ __forceinline__ float mean_x(const RowStat& r) { return r.t / r.s - kExpBias; }
// 16 bytes of the gradient. kEntropy: with the term in x.
template <class T, bool kEntropy>
__device__ __forceinline__ void emit(const uint4& q, const RowGrad& c, float k, F2 (&v)[Elt<T>::W / 2]) {
    Elt<T>::pairs(q, v);
    const F2 k2 = f2_dup(k), neg = f2_dup(-c.m), c0 = f2_dup(c.c0), c1 = f2_dup(c.c1),
             bias = f2_dup(kExpBias);
#pragma unroll
    for (int i = 0; i < Elt<T>::W / 2; ++i) {
        const F2 x = f2_fma3(f2_add(v[i], neg), k2, bias), e = f2_exp2(x);
        F2 f = c0;
        if (kEntropy) f2_fma(f, f2_floor_x(x), c1);
        v[i] = f2_mul(e, f);
    }
}
// `by` joins entry i.
template <int P>
__device__ __forceinline__ void add_at(F2 (&v)[P], int i, float by) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const float2 f = f2_split(v[q]);
        v[q] = f2_make(i == 2 * q ? f.x + by : f.x, i == 2 * q + 1 ? f.y + by : f.y);
    }
}
// 16 bytes to a row's entries j .. of which only those in [0, V) are the row's.
template <class T>
__device__ __forceinline__ void store_part(T* g, int j, int V, const uint4& q) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < Elt<T>::W; ++i)
        if (j + i >= 0 && j + i < V) g[i] = Elt<T>::word(w, i);
}

// Entries j .. of a row as 16 bytes, -infinity outside [0, V).
template <class T>
__device__ __forceinline__ uint4 load_part(const T* p, int j, int V) {
    constexpr int W = Elt<T>::W;
    F2 v[W / 2];
#pragma unroll
    for (int q = 0; q < W; q += 2)
        v[q / 2] = f2_make(j + q >= 0 && j + q < V ? Elt<T>::get(p[j + q]) : -INFINITY,
                           j + q + 1 >= 0 && j + q + 1 < V ? Elt<T>::get(p[j + q + 1]) : -INFINITY);
    return Elt<T>::pack(v);
}

// ln p of the entry with logit z, (z - m) / T - ln S, and in *rest what its rounding leaves.
// The difference, the product and 1 / T go in with their errors, and so does what k's
// rounding to fp32 does to every row's ln S, dk times the mean of x: a sequence adds up
// what all its rows have in common, and beside ln S alone these are below half a unit.
__device__ __forceinline__ float log_prob(const TokenArgs& a, const RowStat& r, float z, float* rest = nullptr) {
    const float y = __fsub_rn(z, r.m), u = __fsub_rn(y, z);
    const float ye = __fsub_rn(__fsub_rn(z, __fsub_rn(y, u)), __fadd_rn(r.m, u));        // z - m = y + ye
    const float p = __fmul_rn(y, a.inv_t), pe = fmaf(y, a.inv_t, -p);
    const float ls = logf(r.s), d = __fsub_rn(p, ls), v = __fsub_rn(d, p);
    const float de = __fsub_rn(__fsub_rn(p, __fsub_rn(d, v)), __fadd_rn(ls, v));         // p - ls = d + de
    const float small = (de + pe) + fmaf(y, a.inv_t_lo, fmaf(ye, a.inv_t, -a.dk * mean_x(r)));
    const bool finite = fabsf(d) < INFINITY;
    const float out = finite ? d + small : d;
    if (rest) *rest = finite ? __fadd_rn(__fsub_rn(d, out), small) : 0.f;
    return out;
}
__device__ __forceinline__ float row_entropy(const RowStat& r) {
    return logf(r.s) - kLn2 * mean_x(r);
}

struct PpoRow {
    float old, adv, ref;
};
__device__ __forceinline__ PpoRow ppo_load(const TokenArgs& a, int64_t row) {
    return PpoRow{a.old_logp[row], a.adv[row], a.ref ? a.ref[row] : 0.f};
}

// The clipped policy loss of one row (l, before its weight) and its gradient.
__device__ __forceinline__ RowGrad ppo_row(const TokenArgs& a, const PpoRow& in, const RowStat& r, float logp, float w,
                                           float* loss, float* clipped, float* kl, float* H) {
    const float A = in.adv;
    const float rho = expf(logp - in.old);
    // an advantage of 0 makes 0 of every ratio, also of one past fp32; a NaN ratio stays one
    const float free_ = A == 0.f && rho == INFINITY ? 0.f : rho * A;
    // a NaN ratio stays one (fminf and fmaxf would drop it)
    const float cut = (rho < a.ratio_lo ? a.ratio_lo : rho > a.ratio_hi ? a.ratio_hi : rho) * A;
    const bool clip = free_ > cut;                   // ties to the unclipped term, which carries the gradient
    *H = row_entropy(r);
    float l = -(clip ? cut : free_) - a.ent * *H;
    float slope = clip ? 0.f : -free_;               // d l / d ln p of the token
    *kl = 0.f;
    if (a.ref) {
        const float d = in.ref - logp, e = expm1f(d);
        *kl = e < INFINITY ? e - d : e;              // e^r outgrows r: +infinity, also at r = +infinity
        if (a.kl != 0.f) {                           // a term that is only reported adds 0, also where e is infinite
            l = fmaf(a.kl, *kl, l);
            slope = fmaf(-a.kl, e, slope);
        }
    }
    *loss = l;
    *clipped = clip ? 1.f : 0.f;
    const float f = w * a.gscale * a.inv_t;
    const float gt = f * slope, h = f * a.ent, inv_s = 1.f / r.s;
    // p (-gt + h (ln p + H)),  ln p = x ln 2 - ln S
    return RowGrad{r.m, inv_s * (a.ent != 0.f ? fmaf(h, *H - logf(r.s), -gt) : -gt), inv_s * h * kLn2, gt};
}

// The gradient of a row whose loss has the slopes `total` at its log-probabilities (the token's and
// the listed entries' together) and `e` at its entropy, before what each of these entries adds, `at`
// times its own slope:
//   d L / d z_j = (1 / T) [ own slope of j - p_j total - e p_j (ln p_j + H) ].
// It goes the losses' way, reading and writing once: memory bounds it (4,096 x 32,768 bf16 with slopes at H 79 us,
// 1,111 x 50,001 fp32 with 64 listed entries 83 us, 69 and 66 at the measured copy's rate).
__device__ __forceinline__ RowGrad scores_row(const TokenArgs& a, float total, float e, const RowStat& r) {
    const float f = a.gscale * a.inv_t, gt = f * total, h = -f * e, inv_s = 1.f / r.s;
    // (an infinite slope at H makes infinities of both signs, and 0 times infinity: the row is NaN)
    const float c0 = e == 0.f ? -gt : fabsf(h) < INFINITY ? fmaf(h, row_entropy(r) - logf(r.s), -gt) : NAN;
    return RowGrad{r.m, inv_s * c0, inv_s * h * kLn2, f};
}

// What a gradient of scores takes besides its list: the slopes at the token's ln p and at H.
struct Slopes {
    float g, e;
};
template <int kOp>
__device__ __forceinline__ Slopes load_slopes(const TokenArgs& a, int64_t row) {
    if (kOp != kTokScores && kOp != kTokScoresList) return Slopes{0.f, 0.f};
    return Slopes{kOp == kTokScores && a.logp_grad ? a.logp_grad[row] : 0.f, a.entropy_grad ? a.entropy_grad[row] : 0.f};
}

// The outputs of a row whose log-probability is all that is asked for.
__device__ __forceinline__ void logp_row(const TokenArgs& a, int64_t row, bool live, const RowStat& r, float z) {
    float rest = 0.f;
    const float logp = live ? log_prob(a, r, z, &rest) : 0.f;
    if (a.logp) a.logp[row] = logp;
    if (a.entropy) a.entropy[row] = live ? row_entropy(r) : 0.f;
    if (a.rows) a.rows[row] = TokenRow{r.m, live ? 1.f / r.s : 0.f, logp, rest};
}

// The statistics of rows: policy loss: KL and H in x, y; distillation: l in x.
struct __align__(16) Totals {
    uint32_t rows, clipped;                          // (64 bits here cost 2 % of 20,000 rows of 300 entries)
    Sum2 loss, x, y;
    __device__ __forceinline__ void add(const RowSum& r) {
        rows += r.flags & 1;
        clipped += r.flags >> 1;
        loss.add(r.loss);
        x.add(r.x);
        y.add(r.y);
    }
    __device__ __forceinline__ void add(const Totals& b) {
        rows += b.rows;
        clipped += b.clipped;
        loss.add(b.loss);
        x.add(b.x);
        y.add(b.y);
    }
};
__device__ __forceinline__ Sum2 sum2_xor(const Sum2& v, int o) {
    return Sum2{__shfl_xor_sync(0xffffffffu, v.s, o), __shfl_xor_sync(0xffffffffu, v.e, o)};
}
// The block's totals in thread 0, in a fixed order.
template <int kThreads>
__device__ __forceinline__ Totals block_totals(Totals v) {
    __shared__ Totals part[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Totals b{__shfl_xor_sync(0xffffffffu, v.rows, o), __shfl_xor_sync(0xffffffffu, v.clipped, o),
                       sum2_xor(v.loss, o), sum2_xor(v.x, o), sum2_xor(v.y, o)};
        v.add(b);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kThreads / 32; ++w) v.add(part[w]);
    return v;
}
// The sum of the blocks' totals part[0 .. n), in thread 0 of the calling block.
template <int kThreads>
__device__ __forceinline__ Totals sum_parts(const Totals* part, int n) {
    static_assert(sizeof(Totals) == 32, "two 16-byte loads");
    Totals v{};
    constexpr int kAt = 4;                           // of two loads each, in flight
    for (int i0 = threadIdx.x; i0 < n; i0 += kAt * kThreads) {
        int4 q[kAt][2];
#pragma unroll
        for (int u = 0; u < kAt; ++u)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                q[u][k] = i0 + u * kThreads < n ? __ldcg(reinterpret_cast<const int4*>(part + i0 + u * kThreads) + k)
                                                : make_int4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < kAt; ++u)
            v.add(Totals{(uint32_t)q[u][0].x, (uint32_t)q[u][0].y, Sum2{__int_as_float(q[u][0].z), __int_as_float(q[u][0].w)},
                         Sum2{__int_as_float(q[u][1].x), __int_as_float(q[u][1].y)},
                         Sum2{__int_as_float(q[u][1].z), __int_as_float(q[u][1].w)}});
    }
    return block_totals<kThreads>(v);
}
template <int kOp>
__device__ __forceinline__ void write_stats(const TokenArgs& a, const Totals& v) {
    const float M = v.rows > 0 ? (float)v.rows : 1.f;
    a.stats[0] = (float)v.rows;
    a.stats[1] = v.loss.value();
    if (kOp == kTokPpo) {
        a.stats[2] = (float)v.clipped / M;
        a.stats[3] = v.x.value() / M;
        a.stats[4] = v.y.value() / M;
    } else {
        a.stats[2] = v.x.value() / M;
    }
}

// The kernels are launched while the stream's one before still runs. This, at every kernel's
// start, waits until that one is complete and what it wrote is there;
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// this lets the next one be launched, once every CTA has come here: in the kernels of a
// preference call, the others' end is near enough.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Launches a kernel that waits for the stream's previous one itself: what the launch takes
// overlaps that one's end. us a call without and with this: one row of 131,072 entries 7.5
// and 6.5, 102,400 rows of 15 12.2 and 11.0, 4,096 rows of 32,768 85 and 82.5.
template <class... Args, class... Given>
cudaError_t launch_after(void (*kernel)(Args...), unsigned grid, unsigned threads, size_t bytes, cudaStream_t s,
                         const Given&... args) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Args(args)...);
}

// The calling CTA has stored what others will read; whether it is the last of `of` that
// come here. The counter is back at 0 for the next call.
__device__ __forceinline__ bool last_of(unsigned* ticket, unsigned of) {
    __shared__ bool last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicInc(ticket, of - 1) == of - 1;
    }
    __syncthreads();
    if (last) __threadfence();
    return last;
}

// A call's rows (token_pairs.cu), by the kernel that takes their length.
cudaError_t launch_token_rows(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
// Short rows (token_short.cuh), by type.
// Most 16-byte vectors of a short row; longer ones go through the ring, which costs some
// microsecond a row and SM. us, short and ring, bf16: policy loss of 10,000 rows of 4,300
// entries 49 and 73, of 6,000 60 and 74, of 8,000 81 and 80 (2,000 rows: 33 and 27);
// log-probabilities of 16,000 rows of 4,300 entries 35 and 55, of 6,000 47 and 54, of 8,000
// 67 and 55. And of a row whose pair's gradient is taken by a warp: longer ones stream past
// it in parts (the preference call on 8,192 rows of 3,001 entries 42 us by warps, 48 in
// parts, of 4,000 43 and 44, of 6,000 64 and 60). fp32 rows change at the same bytes, which
// was not measured: they have half the entries, and where entries bound a row the change
// could come later.
constexpr int kShortVecs = 768, kShortGradVecs = 512;
cudaError_t launch_token_short_f32(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_short_bf16(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_short_f16(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
// Longer ones (token_ring.cuh).
cudaError_t launch_token_ring_f32(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_ring_bf16(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_ring_f16(const TokenArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_pairs(const TokenArgs& a, int n_sm, cudaStream_t s);

}  // namespace malib
