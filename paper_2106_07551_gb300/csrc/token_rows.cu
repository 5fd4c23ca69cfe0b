// Losses of token policies (token_common.cuh has the mathematics): one CTA takes a row
// at a time, gathers its statistics in a first pass over the row and writes the
// gradient in a second one.
#include "token_common.cuh"
#include "token_top.cuh"

namespace malib {

namespace {

constexpr int kT = 512, kW = kT / 32;

// A row's elements in 16-byte vectors of its address: the first and last may be partial.
template <class T>
struct RowFrame {
    static constexpr int W = Elt<T>::W;
    const T* p;
    int h, nv, V;                                    // elements before the row in its first vector; vectors
    __device__ RowFrame(const T* row, int V_) : p(row), V(V_) {
        h = (int)(((uintptr_t)row & 15u) / sizeof(T));
        nv = (h + V + W - 1) / W;
    }
    // Entries outside the row read as -infinity.
    __device__ __forceinline__ uint4 load(int i) const {
        const int j = i * W - h;
        if (j >= 0 && j + W <= V) return *reinterpret_cast<const uint4*>(p + j);
        return load_part(p, j, V);
    }
};

template <class T>
__device__ __forceinline__ void store_vec(T* g, int j, int V, bool aligned, const uint4& v) {
    constexpr int W = Elt<T>::W;
    if (aligned && j >= 0 && j + W <= V) *reinterpret_cast<uint4*>(g + j) = v;
    else store_part(g + j, j, V, v);
}

template <class T>
__device__ void zero_row(T* g, int V) {
    const RowFrame<T> f(g, V);
    const uint4 z = make_uint4(0, 0, 0, 0);
    for (int i = threadIdx.x; i < f.nv; i += kT) store_vec(g, i * Elt<T>::W - f.h, V, true, z);
}

// The gradient of a whole row (every thread of the block).
template <class T>
__device__ void write_row(const T* z, T* g, int V, float k, const RowGrad& c, int token) {
    constexpr int W = Elt<T>::W;
    const RowFrame<T> f(z, V);
    const bool aligned = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
    for (int i = threadIdx.x; i < f.nv; i += kT) {
        F2 v[W / 2];
        emit<T, true>(f.load(i), c, k, v);
        const int j = i * W - f.h;
        if ((unsigned)(token - j) < (unsigned)W) add_at(v, token - j, c.at);
        store_vec(g, j, V, aligned, Elt<T>::pack(v));
    }
}

template <class T, int kOp>
__global__ void __launch_bounds__(kT) token_rows_kernel(TokenArgs a) {
    __shared__ RowStat red[2][kW];
    __shared__ RowGrad grad;
    __shared__ TopEntry list[kOp == kTokDistill ? kTokenMaxTop : 1];
    __shared__ TopRow top;
    double acc[kTokenStats] = {};                    // thread 0
    int buf = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        T* g = a.g ? static_cast<T*>(a.g) + row * a.gld : nullptr;
        int token = -1;
        bool live = true;
        float w = 1.f;
        if (kOp == kTokDistill) {
            if (threadIdx.x < 32) {
                const TopRow t = top_row<T>(a, row, z, list);
                if (threadIdx.x == 0) top = t;
            }
            __syncthreads();
            live = top.live != 0;
        } else {
            token = a.tokens[row];
            live = token >= 0 && token < a.V;
            if (token >= a.V && threadIdx.x == 0) atomicOr(a.err, ERRBIT_BAD_TOKEN);
        }
        if (kOp != kTokLogp) {
            w = a.weight ? a.weight[row] : a.w0;
            live = live && w != 0.f;
        }
        RowStat r{-INFINITY, 0.f, 0.f};
        if (live) {
            const RowFrame<T> f(z, a.V);
            for (int i = threadIdx.x; i < f.nv; i += kT) {
                const uint4 q[1] = {f.load(i)};
                raise(r, vec_max<T>(q), a.k);
                if (r.m != -INFINITY) gather<T>(r, q, a.k);
            }
            r = block_stat<kW>(r, a.k, red[buf]);
            buf ^= 1;                                // one barrier a row: the other slots next
            live = r.m != -INFINITY;                 // a row without an entry has no distribution
        }
        float loss = 0.f, logp = 0.f, H = 0.f;
        if (threadIdx.x == 0) {
            if (live) {
                acc[0] += 1.0;
                RowGrad c{r.m, 0.f, 0.f, 0.f};
                if (kOp == kTokDistill) {
                    loss = top_loss(a, r, top);
                    c.c0 = w * a.gscale * a.top_scale / r.s;
                    acc[1] += (double)w * loss;
                    acc[2] += loss;
                } else if (kOp == kTokPpo) {
                    logp = log_prob(a, r, Elt<T>::get(z[token]));
                    float clipped, kl;
                    c = ppo_row(a, ppo_load(a, row), r, logp, w, &loss, &clipped, &kl, &H);
                    acc[1] += (double)w * loss;
                    acc[2] += clipped;
                    acc[3] += kl;
                    acc[4] += H;
                }
                grad = c;
            }
            if (kOp == kTokLogp) logp_row(a, row, live, r, live ? Elt<T>::get(z[token]) : 0.f);
            if (kOp == kTokPpo && a.logp) a.logp[row] = logp;
            if (kOp == kTokDistill && a.loss) a.loss[row] = loss;
        }
        if (kOp == kTokLogp) continue;
        __syncthreads();
        if (g) {
            if (!live) {
                zero_row(g, a.V);
            } else if (kOp == kTokPpo) {
                write_row(z, g, a.V, a.k, grad, token);
            } else {
                // the teacher's entries go over what the row's threads have written
                const RowGrad c = grad;
                write_row(z, g, a.V, a.k, c, -1);
                __syncthreads();
                for (int j = threadIdx.x; j < a.top; j += kT) {
                    const TopEntry t = list[j];
                    if (t.id >= 0)
                        g[t.id] = Elt<T>::put(c.c0 * exp2_fast((t.z - c.m) * a.k) - w * a.gscale * a.top_scale * t.q);
                }
            }
        }
        __syncthreads();                             // grad and list are free
    }
    if (kOp == kTokLogp || !a.stats) return;
    double v[kTokenStats];
    if (!sum_partials<kT>(a.part, a.ticket, acc, v)) return;
    if (kOp == kTokPpo) {
        ppo_stats(a, v);
    } else {
        distill_stats(a, v);
    }
}

constexpr int kPairT = 128;

// One CTA a pair: the rewards of its two sequences, the loss, and the factor of its
// rows' gradients. Sums in fp64, in a fixed order.
__global__ void __launch_bounds__(kPairT) token_pairs_kernel(TokenArgs a) {
    __shared__ double red[kPairT / 32];
    double acc[kTokenStats] = {};
    for (int p = blockIdx.x; p < a.n_pairs; p += gridDim.x) {
        const int64_t o0 = a.offsets[2 * p], o1 = a.offsets[2 * p + 1], o2 = a.offsets[2 * p + 2];
        const bool ok = o0 >= 0 && o0 <= o1 && o1 <= o2 && o2 <= a.n && (p > 0 || o0 == 0) &&
                        (p + 1 < a.n_pairs || o2 == a.n);
        if (!ok && threadIdx.x == 0) atomicOr(a.err, ERRBIT_BAD_OFFSETS);
        float rew[2];
        __shared__ float factor;
        for (int side = 0; side < 2; ++side) {
            const int64_t lo = !ok ? 0 : side ? o1 : o0, hi = !ok ? 0 : side ? o2 : o1;
            double s = 0.0;
            for (int64_t i = lo + threadIdx.x; i < hi; i += kPairT)
                if (a.rows[i].live) s += (double)a.rows[i].value - (a.ref ? (double)a.ref[i] : 0.0);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            __syncthreads();
            if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
            __syncthreads();
            s = 0.0;
            for (int w = 0; w < kPairT / 32; ++w) s += red[w];
            rew[side] = (float)(a.beta * s);
            if (threadIdx.x == 0) {
                if (a.reward) a.reward[2 * p + side] = rew[side];
                acc[3 + side] += a.beta * s;
            }
        }
        if (threadIdx.x == 0) {
            const float d = rew[0] - rew[1];
            // -ln s(x) = max(-x, 0) + ln(1 + e^-|x|)
            const float tail = log1pf(expf(-fabsf(d)));
            const float lp = fmaxf(-d, 0.f) + tail, ln = fmaxf(d, 0.f) + tail;
            acc[0] += 1.0;
            acc[1] += (double)((1.f - a.smooth) * lp + a.smooth * ln);
            acc[2] += d > 0.f ? 1.0 : 0.0;
            // smooth s(d) - (1 - smooth) s(-d)
            const float slope = a.smooth / (1.f + expf(-d)) - (1.f - a.smooth) / (1.f + expf(d));
            factor = slope * a.beta * a.gscale * a.inv_t / (float)a.n_pairs;
        }
        __syncthreads();
        const float f = factor;
        if (a.g && ok) {
            for (int64_t i = o0 + threadIdx.x; i < o2; i += kPairT) a.rows[i].value = i < o1 ? f : -f;
        }
    }
    if (!a.stats) return;
    double v[kTokenStats];
    if (!sum_partials<kPairT>(a.part, a.ticket, acc, v)) return;
    a.stats[0] = (float)v[0];
    for (int i = 1; i < 5; ++i) a.stats[i] = (float)(v[i] / v[0]);
}

template <class T>
cudaError_t launch_rows_t(const TokenArgs& a, int op, int grid, cudaStream_t s) {
    if (op == kTokLogp) token_rows_kernel<T, kTokLogp><<<grid, kT, 0, s>>>(a);
    else if (op == kTokPpo) token_rows_kernel<T, kTokPpo><<<grid, kT, 0, s>>>(a);
    else token_rows_kernel<T, kTokDistill><<<grid, kT, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

// From this many bytes on a row is long: it goes through shared memory (token_ring.cu).
constexpr int kLongBytes = 2048;

cudaError_t launch_token_rows(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    if (a.n > 0 && (int64_t)a.V * (a.dtype == MALIB_F32 ? 4 : 2) >= kLongBytes) return launch_token_ring(a, op, n_sm, s);
    const int grid = (int)(a.n < 4 * (int64_t)n_sm ? (a.n > 0 ? a.n : 1) : 4 * (int64_t)n_sm);
    if (a.dtype == MALIB_F32) return launch_rows_t<float>(a, op, grid, s);
    if (a.dtype == MALIB_BF16) return launch_rows_t<__nv_bfloat16>(a, op, grid, s);
    return launch_rows_t<__half>(a, op, grid, s);
}

cudaError_t launch_token_pairs(const TokenArgs& a, int n_sm, cudaStream_t s) {
    cudaError_t e = a.n > 0 ? launch_token_rows(a, kTokLogp, n_sm, s) : cudaSuccess;
    if (e != cudaSuccess) return e;
    token_pairs_kernel<<<a.n_pairs < 4 * n_sm ? a.n_pairs : 4 * n_sm, kPairT, 0, s>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess || !a.g || a.n == 0) return e;
    return launch_token_pair_grad(a, s);
}

}  // namespace malib
