// Losses of token policies: which kernel takes a call's rows, and the preference loss of
// answer pairs between its rows' statistics and their gradients.
#include "token_common.cuh"
#include "token_shift.cuh"

namespace malib {

namespace {

constexpr int kPairT = 256;

__device__ __forceinline__ Sum2 warp_sum2(Sum2 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v.add(sum2_xor(v, o));
    return v;
}

// One CTA a pair: the rewards of its two sequences, the loss, and the factor of its
// rows' gradients. Bound by latency (four rows' 16 bytes a thread from L2, sums, a logarithm;
// a call on one pair of 100,000 rows of 15 entries takes 113 us, most of them here): some 5 us
// between the kernels before and after it, which are launched while it and the statistics
// run (333 rows of 4 pairs 24 us a call without that, 22 with it, 19 where the call's first
// kernel overlaps the stream's one before as well).
__global__ void __launch_bounds__(kPairT) token_pairs_kernel(TokenArgs a) {
    __shared__ Sum2 red[kPairT / 32];
    __shared__ float factor;
    constexpr int kHalf = kPairT / 2;
    const int side = threadIdx.x / kHalf, part = threadIdx.x % kHalf;
    Totals total{};                                  // thread 0: pairs, those in order; loss, rewards
    constexpr int kSettle = 1024;                    // rows, pairs after which a sum is settled
    constexpr int kLoads = 4;                        // of a thread in flight
    unsigned taken = 0;
    wait_for_previous();
    let_next_start();
    for (int64_t p = blockIdx.x; p < a.n_pairs; p += gridDim.x) {          // 2 p + 2 passes 31 bits at 2^30 pairs
        const int64_t o0 = a.offsets[2 * p], o1 = a.offsets[2 * p + 1], o2 = a.offsets[2 * p + 2];
        const bool ok = o0 >= 0 && o0 <= o1 && o1 <= o2 && o2 <= a.n && (p > 0 || o0 == 0) &&
                        (p + 1 < a.n_pairs || o2 == a.n);
        if (!ok && threadIdx.x == 0) atomicOr(a.err, ERRBIT_BAD_OFFSETS);
        const int64_t lo = !ok ? 0 : side ? o1 : o0, hi = !ok ? 0 : side ? o2 : o1;
        Sum2 s{0.f, 0.f};
        for (int64_t i0 = lo + part; i0 < hi; i0 += kSettle * kHalf) {
            const TokenRow* rows = a.rows + i0;
            const float* ref = a.ref ? a.ref + i0 : nullptr;
            const int n = (int)min((int64_t)kSettle, (hi - i0 + kHalf - 1) / kHalf);
            for (int u0 = 0; u0 < n; u0 += kLoads) {
                float4 r[kLoads];
                float f[kLoads];
#pragma unroll
                for (int u = 0; u < kLoads; ++u) {   // past the end the last one again: no load waits for a branch
                    const int at = min(u0 + u, n - 1) * kHalf;
                    r[u] = __ldcg(reinterpret_cast<const float4*>(rows + at));
                    f[u] = ref ? __ldcg(ref + at) : 0.f;
                }
#pragma unroll
                for (int u = 0; u < kLoads; ++u) {
                    if (u0 + u >= n || r[u].y == 0.f) continue;               // inv_s
                    s.add(r[u].z);
                    s.e += r[u].w;
                    if (ref) s.add(-f[u]);
                }
            }
            s.settle();
        }
        s = warp_sum2(s);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            float rew[2];
            for (int q = 0; q < 2; ++q) {
                Sum2 v = red[q * (kHalf / 32)];
                for (int i = 1; i < kHalf / 32; ++i) v.add(red[q * (kHalf / 32) + i]);
                rew[q] = fmaf(a.beta, v.s, a.beta * (fabsf(v.s) < INFINITY ? v.e : 0.f));
                if (a.reward) a.reward[2 * p + q] = rew[q];
            }
            const float d = rew[0] - rew[1];
            // -ln s(x) = max(-x, 0) + ln(1 + e^-|x|)
            const float tail = log1pf(expf(-fabsf(d)));
            const float lp = fmaxf(-d, 0.f) + tail, ln = fmaxf(d, 0.f) + tail;
            // without smoothing the second term adds 0, also where it is infinite
            const float second = a.smooth != 0.f ? a.smooth * ln : 0.f;
            total.add(RowSum{(1.f - a.smooth) * lp + second, rew[0], rew[1], d > 0.f ? 3 : 1});
            if (++taken % kSettle == 0) {
                total.loss.settle();
                total.x.settle();
                total.y.settle();
            }
            // smooth s(d) - (1 - smooth) s(-d)
            const float slope = a.smooth / (1.f + expf(-d)) - (1.f - a.smooth) / (1.f + expf(d));
            factor = slope * a.beta * a.gscale * a.inv_t / (float)a.n_pairs;
        }
        if (!a.g || !ok) continue;
        __syncthreads();
        const float f = factor;
        for (int64_t i = o0 + threadIdx.x; i < o2; i += kPairT) a.rows[i].value = i < o1 ? f : -f;
    }
    if (!a.stats) return;
    if (threadIdx.x == 0) a.part[blockIdx.x] = total;
    if (!last_of(a.ticket, gridDim.x)) return;
    const Totals v = sum_parts<kPairT>(a.part, (int)gridDim.x);
    if (threadIdx.x != 0) return;
    const float n = (float)a.n_pairs;
    a.stats[0] = n;
    a.stats[1] = v.loss.value() / n;
    a.stats[2] = (float)v.clipped / n;
    a.stats[3] = v.x.value() / n;
    a.stats[4] = v.y.value() / n;
}

constexpr int kGradT = 256, kGradPer = 4, kGradVecs = kGradT * kGradPer;

// The gradient of preference pairs from the rows' statistics and factors: a CTA per part
// of a row, entries straight from and to global memory, as a copy would go: 6.8 TB/s at
// 2,048 rows of 65,536 bf16 entries, bound by memory. Nothing has to stay on chip here, and
// small CTAs keep more loads in flight than the ring does.
template <class T>
__global__ void __launch_bounds__(kGradT) token_pair_grad_kernel(TokenArgs a, int parts) {
    constexpr int W = Elt<T>::W;
    const int tid = threadIdx.x;
    const int64_t total = a.n * parts;
    wait_for_previous();
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int64_t at = total - 1 - i, row = at / parts;        // the rows read last may still be in the L2 cache
        const int v0 = (int)(at - row * parts) * kGradVecs;
        const TokenRow r = a.rows[row];
        const int token = a.tokens[row];
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        T* g = static_cast<T*>(a.g) + row * a.gld;
        const int h = (int)(((uintptr_t)g & 15u) / sizeof(T));       // vectors of the gradient's own alignment
        const int zo = (int)((uintptr_t)z & 15u) - (int)((uintptr_t)g & 15u);
        const RowGrad c{r.m, -r.value * r.inv_s, 0.f, r.value};
        uint4 q[kGradPer];
#pragma unroll
        for (int u = 0; u < kGradPer; ++u) {
            const int j = (v0 + tid + u * kGradT) * W - h;
            q[u] = Elt<T>::none();
            if (r.inv_s == 0.f || j >= a.V) continue;
            if (zo == 0 && j >= 0 && j + W <= a.V) {
                q[u] = __ldcs(reinterpret_cast<const uint4*>(z + j));
            } else {
                // a vector that starts inside one of the logits' blocks, or a partial one
                const uint8_t* p = reinterpret_cast<const uint8_t*>(z + j);
                const int by = (int)((uintptr_t)p & 15u);
                if (j - W >= 0 && j + 2 * W <= a.V) q[u] = by ? load_shifted(p - by, by) : *reinterpret_cast<const uint4*>(p);
                else q[u] = load_part(z, j, a.V);
            }
        }
#pragma unroll
        for (int u = 0; u < kGradPer; ++u) {
            const int j = (v0 + tid + u * kGradT) * W - h;
            if (j >= a.V) continue;
            F2 v[W / 2];
            emit<T, false>(q[u], c, a.k, v);
            if ((unsigned)(token - j) < (unsigned)W) add_at(v, token - j, c.at);
            uint4 out = Elt<T>::pack(v);
            if (r.inv_s == 0.f) out = make_uint4(0, 0, 0, 0);
            if (j >= 0 && j + W <= a.V) __stcs(reinterpret_cast<uint4*>(g + j), out);
            else store_part(g + j, j, a.V, out);
        }
    }
}

bool is_short(const TokenArgs& a, int op) {
    const int W = a.dtype == MALIB_F32 ? 4 : 8;
    return (a.V + 2 * (int64_t)W - 2) / W <= (op == kTokPairGrad ? kShortGradVecs : kShortVecs);
}

cudaError_t launch_short(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    if (a.dtype == MALIB_F32) return launch_token_short_f32(a, op, n_sm, s);
    if (a.dtype == MALIB_BF16) return launch_token_short_bf16(a, op, n_sm, s);
    return launch_token_short_f16(a, op, n_sm, s);
}

cudaError_t launch_ring(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    if (a.dtype == MALIB_F32) return launch_token_ring_f32(a, op, n_sm, s);
    if (a.dtype == MALIB_BF16) return launch_token_ring_bf16(a, op, n_sm, s);
    return launch_token_ring_f16(a, op, n_sm, s);
}

cudaError_t launch_pair_grad(const TokenArgs& a, cudaStream_t s) {
    const int W = a.dtype == MALIB_F32 ? 4 : 8;
    const int parts = (int)(((a.V + 2 * (int64_t)W - 2) / W + kGradVecs - 1) / kGradVecs);
    const int64_t total = a.n * parts;
    const unsigned grid = (unsigned)(total < (1 << 30) ? total : (1 << 30));
    if (a.dtype == MALIB_F32) return launch_after(token_pair_grad_kernel<float>, grid, kGradT, 0, s, a, parts);
    if (a.dtype == MALIB_BF16) return launch_after(token_pair_grad_kernel<__nv_bfloat16>, grid, kGradT, 0, s, a, parts);
    return launch_after(token_pair_grad_kernel<__half>, grid, kGradT, 0, s, a, parts);
}

}  // namespace

cudaError_t launch_token_rows(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    if (a.n == 0) {
        // No rows: the statistics of none, written by a kernel whose launch does not go by the vocabulary.
        TokenArgs none = a;
        none.V = 1;
        return a.stats ? launch_short(none, op, n_sm, s) : cudaSuccess;
    }
    return is_short(a, op) ? launch_short(a, op, n_sm, s) : launch_ring(a, op, n_sm, s);
}

cudaError_t launch_token_pairs(const TokenArgs& a, int n_sm, cudaStream_t s) {
    cudaError_t e = a.n > 0 ? launch_token_rows(a, kTokLogp, n_sm, s) : cudaSuccess;
    if (e != cudaSuccess) return e;
    e = launch_after(token_pairs_kernel, (unsigned)(a.n_pairs < 4 * n_sm ? a.n_pairs : 4 * n_sm), kPairT, 0, s, a);
    if (e != cudaSuccess || !a.g || a.n == 0) return e;
    return is_short(a, kTokPairGrad) ? launch_short(a, kTokPairGrad, n_sm, s) : launch_pair_grad(a, s);
}

}  // namespace malib
