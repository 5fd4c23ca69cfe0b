// Losses of token policies, long rows: one pass over memory. A row is read from global
// memory once; it stays in shared memory while its statistics are gathered, and the
// gradient is computed from there.
//
// A cluster of C CTAs takes a row, each a slice of it. One warp of a CTA (the producer)
// runs ahead and copies slices into a ring of 16 KB stages with bulk copies, completing
// on an mbarrier per stage; eight warps (the consumers) gather the slice's statistics
// stage by stage, exchange them with the row's other CTAs through distributed shared
// memory (asynchronous stores that complete on an mbarrier), and go through the same
// stages again, writing the gradient to global memory and freeing each stage as they
// leave it. The next row's copies fill the freed stages meanwhile.
//
// Bound by memory: the ring of two CTAs an SM holds 2 x 96 KB in flight or in work, and
// a CTA that waits for its row's sums leaves the SM's other CTA to compute. Per entry
// the first sweep takes about 6 issue slots and one exponential, the second 5 and
// another one, where the memory's rate leaves about 21 a 16-bit entry (read and written)
// and twice that a 32-bit one.
//
// Rows start at any element: a row's vectors are the 16-byte blocks of its address, the
// full ones copied in bulk, a partial first or last one filled in by the producer's
// lanes with -infinity outside the row. Where logits and gradient rows are aligned alike
// (mod 16 bytes) the gradient is written in vectors, otherwise entry by entry with
// consecutive lanes on consecutive entries.
#include <mutex>

#include "token_common.cuh"
#include "token_peer.cuh"

namespace malib {

namespace {

constexpr int kConsumers = 256, kConsumerWarps = kConsumers / 32;
constexpr int kPer = 4;                              // vectors a thread and stage
constexpr int kStageVecs = kPer * kConsumers, kStageBytes = kStageVecs * 16;
constexpr int kMaxStages = 13, kMaxCluster = 8;

// A stage of nothing but full vectors, the row's token not among them.
template <class T, bool kEntropy>
__device__ __forceinline__ void emit_stage(const uint4* q, T* out, const RowGrad& c, float k) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        F2 v[Elt<T>::W / 2];
        emit<T, kEntropy>(q[u * kConsumers], c, k, v);
        __stcs(reinterpret_cast<uint4*>(out + u * kConsumers * Elt<T>::W), Elt<T>::pack(v));
    }
}

__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory"); }

// What the row's CTAs exchange, and what a warp leaves for its CTA.
struct __align__(16) Partial {
    float m, s, t, z;                                // z: the logit of the row's token
};

// A place in the ring: the stage and the parity of its present use.
struct Cursor {
    int stage = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++stage == stages) {
            stage = 0;
            parity ^= 1u;
        }
    }
};

struct Shape {
    int cluster, stages;                             // CTAs a row, stages a CTA
    int slice;                                       // vectors of a CTA's slice
};

// A row's scalars.
struct RowIn {
    int token;
    float w;
    PpoRow ppo;
    TokenRow row;
};
template <int kOp>
__device__ __forceinline__ RowIn load_row(const TokenArgs& a, int64_t row) {
    RowIn in{};
    in.token = a.tokens[row];
    in.w = kOp == kTokPpo ? (a.weight ? a.weight[row] : a.w0) : 1.f;
    if (kOp == kTokPpo) in.ppo = ppo_load(a, row);
    if (kOp == kTokPairGrad) in.row = a.rows[row];
    return in;
}

template <class T, int kOp>
__global__ void __launch_bounds__(kConsumers + 32, kOp == kTokLogp ? 3 : 2) token_ring_kernel(TokenArgs a, Shape sh) {
    constexpr int W = Elt<T>::W;
    constexpr int kThreads = kConsumers + 32;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], xbar[2];
    __shared__ Partial red[2][kConsumerWarps], xslot[2][kMaxCluster];
    __shared__ int dead;                             // a bounded wait has expired: nothing waits any more
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = sh.cluster, rank = C > 1 ? (int)cluster_rank() : 0;
    const int64_t first = blockIdx.x / C, step = gridDim.x / C;
    const int v_lo = rank * sh.slice;

    if (tid == 0) {
        dead = 0;
        for (int i = 0; i < sh.stages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], kConsumerWarps);
        }
        mbar_init(&xbar[0], 1);
        mbar_init(&xbar[1], 1);
        fence_proxy_async_smem();
    }
    __syncthreads();
    if (C > 1) {
        // the peers' barriers and memory are there before the first store to them
        cluster_arrive();
        cluster_wait();
    }
    volatile int* gone = &dead;
    auto expired = [&] {
        *gone = 1;
        atomicOr(a.err, ERRBIT_TIMEOUT);
    };
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (mbar_try_wait(bar, parity) || *gone) return;
        if (!mbar_wait_bounded(bar, parity, kWaitLimitNs)) expired();
    };
    // Whether a row's logits are read: known from its token and weight alone.
    auto wanted = [&](int token, float w) { return token >= 0 && token < a.V && w != 0.f; };
    double acc[kTokenStats] = {};

    if (warp == kConsumerWarps) {
        // ---- producer
        const T* z0 = static_cast<const T*>(a.z);
        Cursor at, issued;
        bool wrapped = false;
        for (int64_t base = first; base < a.n; base += 32 * step) {
            const int64_t mine = base + lane * step;
            bool want = false;
            if (mine < a.n) {
                if (kOp == kTokPairGrad) want = a.rows[mine].live != 0;
                else want = wanted(a.tokens[mine], kOp == kTokLogp ? 1.f : a.weight ? a.weight[mine] : a.w0);
            }
            unsigned todo = __ballot_sync(0xffffffffu, want);
            while (todo) {
                const int64_t row = base + (__ffs(todo) - 1) * step;
                todo &= todo - 1;
                const T* z = z0 + row * a.ld;
                const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
                const int hi = min(nv, v_lo + sh.slice);
                for (int v = v_lo; v < hi; v += kStageVecs, at.next(sh.stages)) {
                    const int n = min(kStageVecs, hi - v), stage = at.stage;
                    uint8_t* dst = ring + stage * kStageBytes;
                    // a partial first (lanes 0..7) or last (lanes 16..23) vector of the row
                    const bool head = v == 0 && h > 0, tail = v + n == nv && (h + a.V) % W != 0;
                    const int pv = lane < 16 ? 0 : nv - 1, pj = pv * W - h + (lane & 15);
                    const bool fill = (lane & 15) < W && (lane < 16 ? head : tail);
                    T part = Elt<T>::put(-INFINITY);
                    if (fill && pj >= 0 && pj < a.V) part = z[pj];
                    wait(&empty[stage], at.parity ^ 1u);
                    if (fill) reinterpret_cast<T*>(dst)[(pv - v) * W + (lane & 15)] = part;
                    __syncwarp();
                    if (*gone) continue;
                    wrapped |= stage + 1 == sh.stages;
                    issued = at;
                    if (lane == 0) {
                        const int b0 = head ? 1 : 0, b1 = tail ? n - 1 : n;
                        const uint32_t bytes = b1 > b0 ? (uint32_t)(b1 - b0) * 16u : 0u;
                        mbar_arrive_expect_tx(&full[stage], bytes);
                        if (bytes) bulk_g2s(dst + b0 * 16, z + ((int64_t)(v + b0) * W - h), bytes, &full[stage]);
                    }
                    __syncwarp();
                }
            }
        }
        if (*gone)                                   // copies in flight end before the block does
            for (int i = 0; i < sh.stages; ++i)
                if (i <= issued.stage || wrapped)
                    mbar_wait_bounded(&full[i], i <= issued.stage ? issued.parity : issued.parity ^ 1u, 1000000);
    } else {
        // ---- consumers
        Cursor at;
        uint32_t exch = 0;
        // a row's scalars are read while the row before is worked on
        RowIn next = load_row<kOp>(a, first);
        for (int64_t row = first; row < a.n; row += step) {
            const RowIn in = next;
            if (row + step < a.n) next = load_row<kOp>(a, row + step);
            const T* z = static_cast<const T*>(a.z) + row * a.ld;
            T* g = kOp != kTokLogp && a.g ? static_cast<T*>(a.g) + row * a.gld : nullptr;
            const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
            const int v_hi = max(v_lo, min(nv, v_lo + sh.slice));
            const int token = in.token;
            const float w = in.w;
            // whether the row's logits are read, and then whether it has a distribution
            const bool read = kOp == kTokPairGrad ? in.row.live != 0 : wanted(token, w);
            bool live = read;
            RowGrad c{0.f, 0.f, 0.f, 0.f};
            const Cursor begin = at;
            if (kOp == kTokPairGrad) {
                c = RowGrad{in.row.m, -in.row.value * in.row.inv_s, 0.f, in.row.value};
            } else {
                if (token >= a.V && rank == 0 && tid == 0) atomicOr(a.err, ERRBIT_BAD_TOKEN);
                RowStat r{-INFINITY, 0.f, 0.f};
                float zt = 0.f;
                if (read) {
                    if (tid == 0) zt = Elt<T>::get(z[token]);
                    for (int v = v_lo; v < v_hi; v += kStageVecs, at.next(sh.stages)) {
                        const int n = min(kStageVecs, v_hi - v), stage = at.stage;
                        const uint4* src = reinterpret_cast<const uint4*>(ring + stage * kStageBytes);
                        wait(&full[stage], at.parity);
                        if (n == kStageVecs) {
                            uint4 q[kPer];
#pragma unroll
                            for (int u = 0; u < kPer; ++u) q[u] = src[tid + u * kConsumers];
                            float mx = Elt<T>::max(q[0]);
#pragma unroll
                            for (int u = 1; u < kPer; ++u) mx = max_nan(mx, Elt<T>::max(q[u]));
                            raise(r, mx, a.k);
                            if (r.m != -INFINITY) {
#pragma unroll
                                for (int u = 0; u < kPer; ++u) gather<T>(r, q[u], a.k);
                            }
                        } else {
                            for (int i = tid; i < n; i += kConsumers) {
                                const uint4 q = src[i];
                                raise(r, Elt<T>::max(q), a.k);
                                if (r.m != -INFINITY) gather<T>(r, q, a.k);
                            }
                        }
                        if (!g) {                    // the slice is not read again
                            __syncwarp();
                            if (lane == 0) mbar_arrive_release(&empty[stage]);
                        }
                    }
                    r = reduce_stat<32>(r, a.k);
                    // the token's logit goes through warp 0's entry: it has been read before
                    // any of the row is written
                    const int slot = exch & 1u;
                    if (lane == 0) red[slot][warp] = Partial{r.m, r.s, r.t, zt};
                    consumer_sync();
                    if (C > 1) {
                        // Two slots are enough: a peer fills this one again only after this
                        // CTA's sums of the next row, which every thread here joins first.
                        if (warp == 0) {
                            const Partial& pw = red[slot][lane & (kConsumerWarps - 1)];
                            r = reduce_stat<kConsumerWarps>(RowStat{pw.m, pw.s, pw.t}, a.k);
                            if (lane == 0) mbar_arrive_expect_tx(&xbar[slot], (uint32_t)(C * sizeof(Partial)));
                            if (lane < C) peer_store(&xslot[slot][rank], &xbar[slot], lane, make_float4(r.m, r.s, r.t, zt));
                        }
                        if (!*gone && !peer_wait_bounded(&xbar[slot], exch >> 1 & 1u, kWaitLimitNs)) expired();
                    }
                    if (C > 1) {
                        const Partial& px = xslot[slot][lane & (kMaxCluster - 1)];
                        r = reduce_stat<kMaxCluster>(
                            lane % kMaxCluster < C ? RowStat{px.m, px.s, px.t} : RowStat{-INFINITY, 0.f, 0.f}, a.k);
                    } else {
                        const Partial& pw = red[slot][lane & (kConsumerWarps - 1)];
                        r = reduce_stat<kConsumerWarps>(RowStat{pw.m, pw.s, pw.t}, a.k);
                    }
                    zt = red[slot][0].z;
                    ++exch;
                    live = r.m != -INFINITY;
                }
                if (kOp == kTokLogp) {
                    if (tid == 0 && rank == 0) logp_row(a, row, live, r, zt);
                    continue;
                }
                float logp = 0.f;
                if (live) {
                    float loss, clipped, kl, H;
                    logp = log_prob(a, r, zt);
                    c = ppo_row(a, in.ppo, r, logp, w, &loss, &clipped, &kl, &H);
                    if (tid == 0 && rank == 0) {
                        acc[0] += 1.0;
                        acc[1] += (double)w * loss;
                        acc[2] += clipped;
                        acc[3] += kl;
                        acc[4] += H;
                    }
                }
                if (a.logp && tid == 0 && rank == 0) a.logp[row] = logp;
            }
            if (!g) continue;
            // the slice again: the gradient
            const bool alike = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
            at = begin;
            for (int v = v_lo; v < v_hi; v += kStageVecs) {
                const int n = min(kStageVecs, v_hi - v);
                const uint8_t* src = ring + at.stage * kStageBytes;
                if (kOp == kTokPairGrad && read) wait(&full[at.stage], at.parity);
                if (alike) {
                    // whether the stage has nothing but full vectors of the row, and not its token
                    const int j_lo = v * W - h;
                    const bool inner = n == kStageVecs && j_lo >= 0 && j_lo + kStageVecs * W <= a.V &&
                                       (unsigned)(token - j_lo) >= (unsigned)(kStageVecs * W);
                    const uint4* q = reinterpret_cast<const uint4*>(src) + tid;
                    T* out = g + (j_lo + tid * W);
                    if (inner && live) {
                        if (kOp == kTokPpo && c.c1 != 0.f) emit_stage<T, true>(q, out, c, a.k);
                        else emit_stage<T, false>(q, out, c, a.k);
                    } else {
                        for (int i = tid; i < n; i += kConsumers, q += kConsumers, out += kConsumers * W) {
                            const int j = j_lo + i * W;
                            F2 x[W / 2] = {};
                            if (live) {
                                emit<T, true>(*q, c, a.k, x);
                                if ((unsigned)(token - j) < (unsigned)W) add_at(x, token - j, c.at);
                            }
                            if (j >= 0 && j + W <= a.V) __stcs(reinterpret_cast<uint4*>(out), Elt<T>::pack(x));
                            else store_part(out, j, a.V, Elt<T>::pack(x));
                        }
                    }
                } else {
                    const int j0 = max(0, v * W - h), j1 = min(a.V, (v + n) * W - h);
                    const T* e0 = reinterpret_cast<const T*>(src) - (v * W - h);
#pragma unroll 4
                    for (int j = j0 + tid; j < j1; j += kConsumers) {
                        float f = 0.f;
                        if (live) {
                            const float x = (Elt<T>::get(e0[j]) - c.m) * a.k;
                            f = exp2_fast(x) * fmaf(c.c1, fmaxf(x, kXMin), c.c0);
                            if (j == token) f += c.at;
                        }
                        g[j] = Elt<T>::put(f);
                    }
                }
                if (read) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(&empty[at.stage]);
                    at.next(sh.stages);
                }
            }
        }
    }
    if (C > 1) {
        // no CTA leaves while a peer may still store to it
        cluster_arrive();
        cluster_wait();
    }
    if (kOp != kTokPpo || !a.stats) return;
    double v[kTokenStats];
    if (!sum_partials<kThreads>(a.part, a.ticket, acc, v)) return;
    ppo_stats(a, v);
}

// CTAs of a kernel that the device holds at once, by cluster size and stages.
template <class T, int kOp>
cudaError_t launch_ring(const TokenArgs& a, const Shape& sh, int per_sm, int n_sm, cudaStream_t s) {
    const void* f = (const void*)token_ring_kernel<T, kOp>;
    const int bytes = sh.stages * kStageBytes;
    cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxStages * kStageBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    cfg.blockDim = dim3(kConsumers + 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    int64_t clusters = (int64_t)per_sm * n_sm;
    if (sh.cluster > 1) {
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = sh.cluster;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        // clusters lie within a part of the device: fewer fit than the SMs' number says
        static std::mutex mu;
        static int held[3][kMaxCluster + 1][kMaxStages + 1];
        static int held_dev = -1;
        int dev = 0;
        if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
        std::lock_guard<std::mutex> lock(mu);
        if (held_dev != dev) {
            for (auto& x : held)
                for (auto& y : x)
                    for (int& q : y) q = 0;
            held_dev = dev;
        }
        int& n = held[per_sm - 1][sh.cluster][sh.stages];
        if (n == 0) {
            cfg.gridDim = dim3(sh.cluster);
            if ((e = cudaOccupancyMaxActiveClusters(&n, f, &cfg)) != cudaSuccess) return e;
            if (n < 1) n = 1;
        }
        clusters = n;
    }
    if (clusters > a.n) clusters = a.n;
    cfg.gridDim = dim3((unsigned)(clusters * sh.cluster));
    e = cudaLaunchKernelEx(&cfg, token_ring_kernel<T, kOp>, a, sh);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <class T>
cudaError_t launch_ring_t(const TokenArgs& a, int op, const Shape& sh, int per_sm, int n_sm, cudaStream_t s) {
    if (op == kTokLogp) return launch_ring<T, kTokLogp>(a, sh, per_sm, n_sm, s);
    if (op == kTokPpo) return launch_ring<T, kTokPpo>(a, sh, per_sm, n_sm, s);
    return launch_ring<T, kTokPairGrad>(a, sh, per_sm, n_sm, s);
}

}  // namespace

bool launch_token_ring(const TokenArgs& a, int op, int n_sm, cudaStream_t s, cudaError_t* e) {
    const int W = a.dtype == MALIB_F32 ? 4 : 8;
    const int64_t nv = (a.V + 2 * (int64_t)W - 2) / W;               // most vectors of a row
    // The smallest cluster that leaves the ring a stage more than a slice; where only
    // the statistics are needed no slice has to stay, and one CTA takes any row.
    const bool whole = op == kTokPpo && a.g;
    Shape sh{1, op == kTokLogp ? 4 : 6, 0};
    int per_sm = op == kTokLogp ? 3 : 2;
    auto slice = [&](int c) { return (nv + c - 1) / c; };
    if (whole) {
        while (sh.cluster < kMaxCluster && slice(sh.cluster) > (sh.stages - 1) * kStageVecs) sh.cluster *= 2;
        if (slice(sh.cluster) > (sh.stages - 1) * kStageVecs) {
            sh.stages = kMaxStages;
            per_sm = 1;
            if (slice(sh.cluster) > kMaxStages * kStageVecs) return false;
        }
    }
    // Few rows: more CTAs a row, down to half a stage.
    while (sh.cluster < kMaxCluster && a.n * sh.cluster * 2 <= (int64_t)per_sm * n_sm &&
           slice(sh.cluster * 2) >= kStageVecs / 2)
        sh.cluster *= 2;
    sh.slice = (int)slice(sh.cluster);
    if (a.dtype == MALIB_F32) *e = launch_ring_t<float>(a, op, sh, per_sm, n_sm, s);
    else if (a.dtype == MALIB_BF16) *e = launch_ring_t<__nv_bfloat16>(a, op, sh, per_sm, n_sm, s);
    else *e = launch_ring_t<__half>(a, op, sh, per_sm, n_sm, s);
    return true;
}

}  // namespace malib
