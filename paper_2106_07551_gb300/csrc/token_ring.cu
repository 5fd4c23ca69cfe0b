// Losses of token policies, long rows: one pass over memory. A row is read from global
// memory once; it stays in shared memory while its statistics are gathered, and the
// gradient is computed from there.
//
// A cluster of C CTAs takes a row, each a slice of it. One warp of a CTA (the producer)
// runs ahead and copies slices into a ring of 16 KB stages with bulk copies, completing
// on an mbarrier per stage; eight warps (the consumers) gather the slice's statistics
// stage by stage; warp 0 exchanges them with the row's other CTAs through distributed
// shared memory (asynchronous stores that complete on an mbarrier) and computes the
// row's loss; and the consumers go through the same stages again, writing the gradient
// to global memory and freeing each stage as they leave it. The next row's copies fill
// the freed stages meanwhile. For distillation a further warp (the teacher) prepares the
// row's list of entries ahead.
//
// Rows are claimed, not dealt: SMs do not all get the same share of the memory's rate, and
// rows that are left out cost a write and no read; with a fixed share each, SMs stood
// idle for 10 to 20% of a call. The producer claims a row ahead (an atomic counter), reads
// its token and weight, and puts it into the CTA's queue. What a row adds to the statistics is stored by itself and summed in the
// rows' order at the end, so that a call's results do not depend on who took what.
//
// Bound by memory: the rings of two CTAs an SM hold 2 x 96 KB in flight or in work, and
// while a CTA waits for its row's sums the SM's other one computes.
//
// Rows start at any element: a row's vectors are the 16-byte blocks of its address, the
// full ones copied in bulk, a partial first or last one filled in by the producer's
// lanes with -infinity outside the row. Where logits and gradient rows are not aligned
// alike (mod 16 bytes) a gradient's vector is put together from two of the ring's.
//
// Every wait is bounded, between the warps too: one that expires ends the CTA's work and
// is reported as MALIB_ETIMEOUT.
#include "token_common.cuh"
#include "token_peer.cuh"
#include "token_top.cuh"

namespace malib {

namespace {

constexpr int kConsumers = 256, kConsumerWarps = kConsumers / 32;
constexpr int kPer = 4;                              // vectors a thread and stage
constexpr int kStageVecs = kPer * kConsumers, kStageBytes = kStageVecs * 16;
constexpr int kMaxStages = 8, kMaxCluster = 8;
constexpr int kQueue = 4;                            // most rows known ahead
constexpr int kRingTwo = 104 * 1024;                 // dynamic shared memory with two CTAs an SM

// What the row's CTAs exchange, and what a warp leaves for its CTA.
struct __align__(16) Partial {
    float m, s, t, unused;
};
// A queued row: token < 0 if it is left out; row < 0 after the last one.
struct __align__(16) Queued {
    int64_t row;
    int32_t token;
    float w;
};
// What warp 0 leaves for the second sweep.
struct RowOut {
    RowGrad c;
    int32_t live;
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
    int keep;                                        // stages that hold parts of a row for its second sweep
    int queue_log, batch;                            // rows known ahead (log 2), rows a claim takes
    int single;                                      // the grid has a CTA, or a cluster, for every row
};

// Sixteen bytes of shared memory from a byte offset that need not be a multiple of 16.
template <int kWord>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, uint32_t bits) {
    const uint32_t w[9] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, 0};
    return make_uint4(__funnelshift_r(w[kWord], w[kWord + 1], bits), __funnelshift_r(w[kWord + 1], w[kWord + 2], bits),
                      __funnelshift_r(w[kWord + 2], w[kWord + 3], bits),
                      __funnelshift_r(w[kWord + 3], w[kWord + 4], bits));
}
__device__ __forceinline__ uint4 load_shifted(const uint8_t* p, int by) {   // p: 16-byte aligned, 0 < by < 16
    const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 16);
    const uint32_t bits = 8u * (by & 3);
    switch (by >> 2) {
        case 0: return shifted<0>(a, b, bits);
        case 1: return shifted<1>(a, b, bits);
        case 2: return shifted<2>(a, b, bits);
        default: return shifted<3>(a, b, bits);
    }
}

// One entry of the gradient.
template <class T>
__device__ __forceinline__ float emit_one(T z, const RowGrad& c, float k) {
    const float x = x_of(Elt<T>::get(z), c.m, k);
    return exp2_fast(x) * fmaf(c.c1, fmaxf(x, kXMin), c.c0);
}

// The gradient of a stage: entries [j0, j1) of the row, those of the n vectors at src,
// the first of which is entry `first` (before the row where the row starts inside it).
template <class T, bool kEntropy>
__device__ __forceinline__ void emit_stage(const uint8_t* src, int first, int j0, int j1, int n, T* g, bool alike,
                                           const RowGrad& c, float k, int token) {
    constexpr int W = Elt<T>::W;
    const int tid = threadIdx.x;
    const T* e = reinterpret_cast<const T*>(src) - first;            // entry j at e[j]
    F2 v[W / 2];
    if (alike) {
        const uint4* q = reinterpret_cast<const uint4*>(src) + tid;
        T* out = g + (first + tid * W);
        if (j0 == first && j1 - j0 == kStageVecs * W) {
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

// Zeros to entries [j0, j1) of a row.
template <class T>
__device__ __forceinline__ void zero_entries(T* g, int j0, int j1) {
    constexpr int W = Elt<T>::W;
    const int tid = threadIdx.x;
    const int to = (int)((16u - ((uintptr_t)(g + j0) & 15u) & 15u) / sizeof(T));
    const int a0 = min(j0 + to, j1), nv = (j1 - a0) / W, a1 = a0 + nv * W;
    for (int i = tid; i < nv; i += kConsumers)
        __stcs(reinterpret_cast<uint4*>(g + (a0 + i * W)), make_uint4(0, 0, 0, 0));
    const int j = tid < W ? j0 + tid : a1 + tid - W;
    if (tid < 2 * W && j < (tid < W ? a0 : j1)) g[j] = Elt<T>::put(0.f);
}

// The statistics of a call from its rows' shares, in the rows' order (every thread of one
// block).
template <int kOp, int kThreads>
__device__ __forceinline__ void sum_rows(const TokenArgs& a) {
    Totals v{};
    constexpr int kAt = 8;                           // loads in flight
    for (int64_t i0 = threadIdx.x; i0 < a.n; i0 += kAt * kThreads) {
        float4 q[kAt];
#pragma unroll
        for (int u = 0; u < kAt; ++u) {
            const int64_t i = i0 + u * kThreads;
            q[u] = i < a.n ? __ldcg(reinterpret_cast<const float4*>(a.row_sums + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < kAt; ++u) v.add(RowSum{q[u].x, q[u].y, q[u].z, __float_as_int(q[u].w)});
    }
    v = block_totals<kThreads>(v);
    if (threadIdx.x == 0) write_stats<kOp>(a, v);
}

template <class T, int kOp>
__global__ void __launch_bounds__(kConsumers + (kOp == kTokDistill ? 64 : 32), kOp == kTokLogp ? 3 : 2)
    token_ring_kernel(TokenArgs a, Shape sh) {
    constexpr int W = Elt<T>::W;
    constexpr int kThreads = kConsumers + (kOp == kTokDistill ? 64 : 32);
    constexpr bool kTop = kOp == kTokDistill;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages];
    // per queued row: known, no longer needed; per row that is read: the warps' statistics
    // are there, the CTAs', the result, the written slice
    __shared__ __align__(8) uint64_t qfull[kQueue], qempty[kQueue], sfull[kQueue], rfull[kQueue], pfull[kQueue],
        xfull;
    __shared__ __align__(8) uint64_t tfull[2], tempty[2];
    __shared__ Queued queue[kQueue];
    __shared__ Partial red[kQueue][kConsumerWarps], xslot[kMaxCluster];
    __shared__ RowOut rout[kQueue];
    constexpr int kSeen = kTop ? 32768 : 32;
    __shared__ uint32_t seen[kSeen / 32];
    __shared__ TopRow top[2];
    __shared__ int dead;                             // a bounded wait has expired: nothing waits any more
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = sh.cluster, rank = C > 1 ? (int)cluster_rank() : 0;
    const int v_lo = rank * sh.slice;
    TopEntry* entries = reinterpret_cast<TopEntry*>(ring + sh.stages * kStageBytes);   // [2][a.top]

    if (tid == 0) {
        dead = 0;
        for (int i = 0; i < sh.stages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], kConsumerWarps);
        }
        for (int i = 0; i < kQueue; ++i) {
            mbar_init(&qfull[i], 1);
            mbar_init(&qempty[i], kThreads / 32);
            mbar_init(&sfull[i], kConsumerWarps);
            mbar_init(&rfull[i], 1);
            mbar_init(&pfull[i], kConsumerWarps);
        }
        mbar_init(&xfull, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&tfull[i], 1);
            mbar_init(&tempty[i], kConsumerWarps);
        }
        fence_proxy_async_smem();
    }
    __syncthreads();
    // The peers' barriers and memory are there before the first store to them: arrived here,
    // waited for where it is needed.
    if (C > 1) cluster_arrive();
    bool joined = C == 1;
    auto join = [&] {
        if (!joined) cluster_wait();
        joined = true;
    };
    volatile int* gone = &dead;
    auto expired = [&] {
        *gone = 1;
        atomicOr(a.err, ERRBIT_TIMEOUT);
    };
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (mbar_try_wait(bar, parity) || *gone) return;
        if (!mbar_wait_bounded(bar, parity, kWaitLimitNs)) expired();
    };
    auto slot_of = [&](uint32_t t) { return t & ((1u << sh.queue_log) - 1u); };
    auto parity_of = [&](uint32_t t) { return t >> sh.queue_log & 1u; };
    // A row's token and weight (row < a.n).
    auto look = [&](int64_t row) {
        Queued q{row, kTop ? 0 : a.tokens[row], 1.f};
        if (kOp != kTokLogp) q.w = a.weight ? a.weight[row] : a.w0;
        return q;
    };
    auto settle = [&](Queued& q, bool report) {
        if (q.token >= a.V && report) atomicOr(a.err, ERRBIT_BAD_TOKEN);
        if (q.token >= a.V || q.w == 0.f) q.token = -1;
    };
    // Turn t's row, as every warp sees it; row < 0: there is none.
    auto take = [&](uint32_t t) {
        Queued q{-1, -1, 0.f};
        if (sh.single) {
            if (t > 0) return q;
            q = look(blockIdx.x / C);
            settle(q, rank == 0 && tid == 0);
            return q;
        }
        wait(&qfull[slot_of(t)], parity_of(t));
        if (!*gone) q = queue[slot_of(t)];
        return q;
    };
    // The warp needs nothing of turn t any more.
    auto leave = [&](uint32_t t) {
        __syncwarp();
        if (lane == 0) mbar_arrive_release(&qempty[slot_of(t)]);
    };

    if (warp == kConsumerWarps) {
        // ---- producer
        // A batch of claimed rows, lane i with the i-th row's token and weight. The next one is
        // claimed (lane 0) when the batch's last row is queued, and looked at when that row's
        // copies are under way: neither is waited for where it is asked for, and no CTA holds
        // rows that another could start on.
        int64_t batch = (int64_t)blockIdx.x * sh.batch;
        int used = 0;
        Queued mine{-1, -1, 0.f};
        auto look_batch = [&] {
            if (lane < sh.batch && batch + lane < a.n) mine = look(batch + lane);
        };
        if (!sh.single) look_batch();
        Cursor at, issued;
        bool wrapped = false;
        for (uint32_t t = 0;; ++t) {
            if (!sh.single) {
                const int slot = slot_of(t);
                Queued q{batch + used < a.n ? batch + used : -1, __shfl_sync(0xffffffffu, mine.token, used),
                         __shfl_sync(0xffffffffu, mine.w, used)};
                if (q.row >= 0) settle(q, lane == 0);
                wait(&qempty[slot], parity_of(t) ^ 1u);
                if (lane == 0) {
                    queue[slot] = q;
                    mbar_arrive_release(&qfull[slot]);
                }
                if (++used == sh.batch && lane == 0)
                    batch = (int64_t)gridDim.x * sh.batch + (int64_t)atomicAdd(a.claims, (unsigned long long)sh.batch);
            }
            const Queued q = take(t);
            if (q.row < 0) break;
            if (q.token >= 0) {
                const T* z = static_cast<const T*>(a.z) + q.row * a.ld;
                const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
                const int hi = max(v_lo, min(nv, v_lo + sh.slice)), parts = (hi - v_lo + kStageVecs - 1) / kStageVecs;
                const int again = kOp != kTokLogp && a.g ? max(0, parts - sh.keep) : 0;
                for (int part = 0; part < parts + again; ++part, at.next(sh.stages)) {
                    const int v = v_lo + (part < parts ? part : part - parts) * kStageVecs;
                    const int n = min(kStageVecs, hi - v), stage = at.stage;
                    uint8_t* dst = ring + stage * kStageBytes;
                    // a partial first (lanes 0..7) or last (lanes 16..23) vector of the row
                    const bool head = v == 0 && h > 0, tail = v + n == nv && (h + a.V) % W != 0;
                    const int pv = lane < 16 ? 0 : nv - 1, pj = pv * W - h + (lane & 15);
                    const bool fill = (lane & 15) < W && (lane < 16 ? head : tail);
                    T entry = Elt<T>::put(-INFINITY);
                    if (fill && pj >= 0 && pj < a.V) entry = z[pj];
                    wait(&empty[stage], at.parity ^ 1u);
                    if (fill) reinterpret_cast<T*>(dst)[(pv - v) * W + (lane & 15)] = entry;
                    __syncwarp();
                    if (*gone) break;
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
            if (!sh.single && used == sh.batch) {
                used = 0;
                batch = __shfl_sync(0xffffffffu, batch, 0);
                look_batch();
            }
            leave(t);
        }
        if (*gone)                                   // copies in flight end before the block does
            for (int i = 0; i < sh.stages; ++i)
                if (wrapped || i <= issued.stage)
                    mbar_wait_bounded(&full[i], i <= issued.stage ? issued.parity : issued.parity ^ 1u, 1000000);
    } else if (warp > kConsumerWarps) {
        // ---- teacher
        if constexpr (kTop) {
            uint32_t turn = 0;                       // rows that are read
            for (uint32_t t = 0;; ++t) {
                const Queued q = take(t);
                if (q.row < 0) break;
                if (q.token >= 0) {
                    const int b = turn & 1u;
                    wait(&tempty[b], (turn >> 1 & 1u) ^ 1u);
                    const TopRow r = top_row<T, kSeen>(a, q.row, static_cast<const T*>(a.z) + q.row * a.ld, entries + b * a.top, seen);
                    if (lane == 0) top[b] = r;
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(&tfull[b]);
                    ++turn;
                }
                leave(t);
            }
        }
    } else {
        // ---- consumers
        Cursor at;
        uint32_t turn = 0;                           // rows that are read
        for (uint32_t t = 0;; ++t) {
            const Queued q = take(t);
            if (q.row < 0) break;
            const int slot = slot_of(turn), b = turn & 1u;
            const uint32_t parity = parity_of(turn);
            const int64_t row = q.row;
            const T* z = static_cast<const T*>(a.z) + row * a.ld;
            T* g = kOp != kTokLogp && a.g ? static_cast<T*>(a.g) + row * a.gld : nullptr;
            const int h = (int)(((uintptr_t)z & 15u) / sizeof(T)), nv = (h + a.V + W - 1) / W;
            const int v_hi = max(v_lo, min(nv, v_lo + sh.slice));
            const bool first = tid == 0 && rank == 0;
            if (q.token < 0) {
                if (first) {
                    if (kOp == kTokLogp) logp_row(a, row, false, RowStat{0.f, 1.f, 0.f}, 0.f);
                    if (kOp == kTokPpo && a.logp) a.logp[row] = 0.f;
                    if (kTop && a.loss) a.loss[row] = 0.f;
                    if (kOp != kTokLogp) a.row_sums[row] = RowSum{0.f, 0.f, 0.f, 0};
                }
                if (g) zero_entries(g, max(0, v_lo * W - h), max(0, min(a.V, v_hi * W - h)));
                leave(t);
                continue;
            }
            T z_token = Elt<T>::put(0.f);            // widened where it is used: nothing waits for it here
            PpoRow in{};
            if (warp == 0) {
                if (!kTop) z_token = z[q.token];
                if (kOp == kTokPpo) in = ppo_load(a, row);
            }
            // the row's last parts stay in the ring, the others come again for the second sweep
            const int parts = (v_hi - v_lo + kStageVecs - 1) / kStageVecs, kept = g ? max(0, parts - sh.keep) : parts;
            Cursor begin;
            RowStat r{-INFINITY, 0.f, 0.f};
            for (int part = 0; part < parts; ++part, at.next(sh.stages)) {
                const int n = min(kStageVecs, v_hi - v_lo - part * kStageVecs);
                if (part == kept) begin = at;
                const uint4* src = reinterpret_cast<const uint4*>(ring + at.stage * kStageBytes);
                wait(&full[at.stage], at.parity);
                uint4 x[kPer];
                if (n == kStageVecs) {
#pragma unroll
                    for (int u = 0; u < kPer; ++u) x[u] = src[tid + u * kConsumers];
                } else {
#pragma unroll
                    for (int u = 0; u < kPer; ++u)
                        x[u] = tid + u * kConsumers < n ? src[tid + u * kConsumers] : Elt<T>::none();
                }
                raise(r, vec_max<T>(x), a.k);
                if (r.m != -INFINITY) gather<T>(r, x, a.k);
                if (part < kept) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(&empty[at.stage]);
                }
            }
            r = reduce_stat<32>(r, a.k);
            if (lane == 0) {
                red[slot][warp] = Partial{r.m, r.s, r.t, 0.f};
                mbar_arrive_release(&sfull[slot]);
            }
            if (warp == 0) {
                wait(&sfull[slot], parity);
                const Partial& pw = red[slot][lane & (kConsumerWarps - 1)];
                r = reduce_stat<kConsumerWarps>(RowStat{pw.m, pw.s, pw.t}, a.k);
                if (kTop) wait(&tfull[b], turn >> 1 & 1u);
                const float zt = Elt<T>::get(z_token);
                if (C > 1) {
                    // The logits that the loss takes (zt, the teacher's entries) have been read
                    // before any CTA of the row writes its part: they go before these sums.
                    join();
                    if (lane == 0) mbar_arrive_expect_tx(&xfull, (uint32_t)(C * sizeof(Partial)));
                    if (lane < C) peer_store(&xslot[rank], &xfull, lane, make_float4(r.m, r.s, r.t, zt));
                    if (!*gone && !peer_wait_bounded(&xfull, 0, kWaitLimitNs)) expired();
                    const Partial& px = xslot[lane & (kMaxCluster - 1)];
                    r = reduce_stat<kMaxCluster>(
                        lane % kMaxCluster < C ? RowStat{px.m, px.s, px.t} : RowStat{-INFINITY, 0.f, 0.f}, a.k);
                }
                bool live = r.m != -INFINITY;
                if (kOp == kTokLogp) {
                    if (first) logp_row(a, row, live, r, zt);
                } else {
                    float loss = 0.f;
                    RowGrad c{0.f, 0.f, 0.f, 0.f};
                    RowSum sum{0.f, 0.f, 0.f, 0};
                    if (kOp == kTokPpo) {
                        float logp = 0.f;
                        if (live) {
                            float clipped, kl, H;
                            logp = log_prob(a, r, zt);
                            c = ppo_row(a, in, r, logp, q.w, &loss, &clipped, &kl, &H);
                            sum = RowSum{q.w * loss, kl, H, clipped != 0.f ? 3 : 1};
                        }
                        if (a.logp && first) a.logp[row] = logp;
                    } else {
                        live = live && top[b].live;
                        if (live) {
                            const float f = q.w * a.gscale * a.top_scale;
                            loss = top_loss(a, r, top[b]);
                            c = RowGrad{r.m, f / r.s, 0.f, f};               // at: the factor of the teacher's q
                            sum = RowSum{q.w * loss, loss, 0.f, 1};
                        }
                        if (a.loss && first) a.loss[row] = loss;
                    }
                    if (first) a.row_sums[row] = sum;
                    if (lane == 0) {
                        rout[slot] = RowOut{c, live};
                        mbar_arrive_release(&rfull[slot]);
                    }
                }
            }
            if (g) {
                wait(&rfull[slot], parity);
                const RowGrad c = rout[slot].c;
                const bool live = rout[slot].live != 0, alike = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
                if (kept < parts) at = begin;
                for (int i = 0; i < parts; ++i, at.next(sh.stages)) {
                    const int part = kept + i < parts ? kept + i : kept + i - parts, v = v_lo + part * kStageVecs;
                    const int n = min(kStageVecs, v_hi - v), j = v * W - h;
                    if (part < kept) wait(&full[at.stage], at.parity);
                    const int j0 = max(0, j), j1 = min(a.V, j + n * W);
                    const uint8_t* src = ring + at.stage * kStageBytes;
                    const int token = kTop ? -1 : q.token;
                    if (!live) zero_entries(g, j0, j1);
                    else if (kOp == kTokPpo && c.c1 != 0.f) emit_stage<T, true>(src, j, j0, j1, n, g, alike, c, a.k, token);
                    else emit_stage<T, false>(src, j, j0, j1, n, g, alike, c, a.k, token);
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(&empty[at.stage]);
                }
                if (kTop) {
                    // the teacher's entries of this slice, over what the CTA's warps have written
                    if (lane == 0) mbar_arrive_release(&pfull[slot]);
                    wait(&pfull[slot], parity);
                    const int j0 = max(0, v_lo * W - h), j1 = min(a.V, v_hi * W - h);
                    if (live)
                        for (int i = tid; i < a.top; i += kConsumers) {
                            const TopEntry e = entries[b * a.top + i];
                            if (e.id >= j0 && e.id < j1)
                                g[e.id] = Elt<T>::put(c.c0 * exp2_fast(x_of(e.z, c.m, a.k)) - c.at * e.q);
                        }
                }
            }
            if (kTop) {
                __syncwarp();
                if (lane == 0) mbar_arrive_release(&tempty[b]);
            }
            ++turn;
            leave(t);
        }
    }
    join();
    if (C > 1) {
        // no CTA leaves while a peer may still store to it
        cluster_arrive();
        cluster_wait();
    }
    // the CTA that ends last clears the claims for the next call and sums the statistics
    const bool stats = kOp != kTokLogp && a.stats;
    if (!stats && sh.single) return;
    if (!last_of(a.ticket, gridDim.x)) return;
    if (tid == 0) *a.claims = 0ull;
    if (stats) sum_rows<kOp, kThreads>(a);
}

// The gradient of preference pairs from the rows' statistics and factors: a CTA per part
// of a row, entries straight from and to global memory, as a copy would go.
template <class T>
__global__ void __launch_bounds__(kConsumers) token_pair_grad_kernel(TokenArgs a, int parts) {
    constexpr int W = Elt<T>::W;
    const int tid = threadIdx.x;
    const int64_t total = a.n * parts;
    for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
        const int64_t row = at / parts;
        const int v0 = (int)(at - row * parts) * kStageVecs;
        const TokenRow r = a.rows[row];
        const int token = a.tokens[row];
        const T* z = static_cast<const T*>(a.z) + row * a.ld;
        T* g = static_cast<T*>(a.g) + row * a.gld;
        const int h = (int)(((uintptr_t)g & 15u) / sizeof(T));       // vectors of the gradient's own alignment
        const int zo = (int)((uintptr_t)z & 15u) - (int)((uintptr_t)g & 15u);
        const RowGrad c{r.m, -r.value * r.inv_s, 0.f, r.value};
        uint4 q[kPer];
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int j = (v0 + tid + u * kConsumers) * W - h;
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
        for (int u = 0; u < kPer; ++u) {
            const int j = (v0 + tid + u * kConsumers) * W - h;
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

template <class T, int kOp>
cudaError_t launch_ring(const TokenArgs& a, const Shape& sh, int grid, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(token_ring_kernel<T, kOp>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingTwo);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kConsumers + (kOp == kTokDistill ? 64 : 32));
    cfg.dynamicSmemBytes = sh.stages * kStageBytes + (kOp == kTokDistill ? 2 * a.top * (int)sizeof(TopEntry) : 0);
    cfg.stream = s;
    if (sh.cluster > 1) {
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = sh.cluster;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
    }
    e = cudaLaunchKernelEx(&cfg, token_ring_kernel<T, kOp>, a, sh);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <class T>
cudaError_t launch_ring_t(const TokenArgs& a, int op, const Shape& sh, int grid, cudaStream_t s) {
    if (op == kTokLogp) return launch_ring<T, kTokLogp>(a, sh, grid, s);
    if (op == kTokPpo) return launch_ring<T, kTokPpo>(a, sh, grid, s);
    return launch_ring<T, kTokDistill>(a, sh, grid, s);
}

}  // namespace

cudaError_t launch_token_ring(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    const int W = a.dtype == MALIB_F32 ? 4 : 8;
    const int64_t nv = (a.V + 2 * (int64_t)W - 2) / W;               // most vectors of a row
    const int lists = op == kTokDistill ? 2 * a.top * (int)sizeof(TopEntry) : 0;
    const int held = (op == kTokLogp ? 3 : 2) * n_sm;                // CTAs the device holds
    Shape sh{1, op == kTokLogp ? 4 : (kRingTwo - lists) / kStageBytes, 0, 0, 0, 1, 0};
    auto slice = [&](int c) { return (nv + c - 1) / c; };
    // CTAs a row: the rounds that the device takes over the rows, times the bytes that a CTA
    // moves in one and what it costs besides (about 4 us, the time of 80 KB). In us, C = 1
    // and the C taken: ppo 25 x 32,768 bf16 20 and 12 (8), distillation 333 x 151,111 fp32
    // 126 and 97 (4); 333 x 32,768 bf16 rows' statistics stay at C = 1, 11, with 4 20.
    const int64_t bytes = a.V * (int64_t)(16 / W) * (op == kTokLogp ? 1 : 2);
    int64_t best = 0;
    for (int c = 1; c <= kMaxCluster && (c == 1 || slice(c) >= kStageVecs / 2); c *= 2) {
        const int64_t t = (a.n * c + held - 1) / held * (80 * 1024 + bytes / c);
        if (c > 1 && t >= best) continue;
        best = t;
        sh.cluster = c;
    }
    sh.slice = (int)slice(sh.cluster);
    sh.keep = sh.slice <= (sh.stages - 1) * kStageVecs ? sh.stages - 1 : sh.stages - 2;
    // A cluster takes one row, as does a CTA when there are no more rows than CTAs.
    sh.single = sh.cluster > 1 || a.n <= held;
    const int64_t grid = sh.single ? a.n * sh.cluster : held;
    // Rows of a stage or more are claimed one by one and known one ahead, so that no CTA holds
    // several while others run out; short ones in batches of about two stages, as long as
    // there are several for every CTA.
    sh.queue_log = sh.slice >= kStageVecs ? 1 : 2;
    if (sh.slice < kStageVecs && !sh.single) {
        const int64_t most = a.n / (4 * grid), about = 2 * kStageVecs / sh.slice;
        sh.batch = (int)(most < 1 ? 1 : most < about ? most : about);
        if (sh.batch > 16) sh.batch = 16;
    }
    if (a.dtype == MALIB_F32) return launch_ring_t<float>(a, op, sh, (int)grid, s);
    if (a.dtype == MALIB_BF16) return launch_ring_t<__nv_bfloat16>(a, op, sh, (int)grid, s);
    return launch_ring_t<__half>(a, op, sh, (int)grid, s);
}

cudaError_t launch_token_pair_grad(const TokenArgs& a, cudaStream_t s) {
    const int W = a.dtype == MALIB_F32 ? 4 : 8;
    const int parts = (int)(((a.V + 2 * (int64_t)W - 2) / W + kStageVecs - 1) / kStageVecs);
    const int64_t total = a.n * parts;
    const unsigned grid = (unsigned)(total < (1 << 30) ? total : (1 << 30));
    if (a.dtype == MALIB_F32) token_pair_grad_kernel<float><<<grid, kConsumers, 0, s>>>(a, parts);
    else if (a.dtype == MALIB_BF16) token_pair_grad_kernel<__nv_bfloat16><<<grid, kConsumers, 0, s>>>(a, parts);
    else token_pair_grad_kernel<__half><<<grid, kConsumers, 0, s>>>(a, parts);
    return cudaGetLastError();
}

}  // namespace malib
