// Losses of token policies, long rows: one pass over memory. A row is read from global
// memory once; it stays in shared memory while its statistics are gathered, and the
// gradient is computed from there. Where a row is longer than the ring, its last parts
// stay and the others are read again, which the L2 cache serves.
//
// One warp of a CTA (the producer) runs ahead and copies rows into a ring of stages with
// bulk copies, completing on an mbarrier per stage; the other warps (the consumers) gather
// a row's statistics stage by stage; warp 0 sums the warps' statistics and computes the
// row's loss; and the consumers go through the same stages again, writing the gradient to
// global memory and freeing each stage as they leave it. The next row's copies fill the
// freed stages meanwhile. For distillation a further warp (the teacher) prepares the row's
// list of entries ahead.
//
// Rows are claimed, not dealt: SMs do not all get the same share of the memory's rate, and
// rows that are left out cost a write and no read; with a fixed share each, SMs stood
// idle for 10 to 20% of a call. The producer claims a row ahead (an atomic counter), reads
// its token and weight, and puts it into the CTA's queue. What a row adds to the
// statistics is stored by itself and summed in the rows' order at the end, so that a
// call's results do not depend on who took what.
//
// With few rows, or very long ones, a cluster of C CTAs takes a row, each a slice of it, and
// exchanges the sums through distributed shared memory (asynchronous stores that complete on
// an mbarrier). Clusters' rows are dealt: a claim would have to be exchanged too.
//
// Bound by memory for rows of 100 KB and more, below by the sweeps' instructions (per entry
// about 7 and an exponential in the first one, 4.5 to 6 and one in the second) and what a
// row costs besides. Stages of 16 KB under four consumer warps with three CTAs an SM, or of
// 32 KB under eight warps: eight vectors a thread and stage hide the latencies of shared
// memory and of the exponential, which four did not. ppo with every term, us a call
// (bf16, 4,096 rows of which a quarter is left out): 64 KB rows 86 with the small shape, 87
// and 113 with two and one CTAs of the large one; 100 KB 130, 136, 166; 128 KB 174, 157,
// 180; 192 KB 287, 254, 249; 16,384 rows of 256 KB 1,648, 1,562, 1,281 (6.4 TB/s).
// Log-probabilities of 8,192 rows of 128 KB, a quarter left out: 119 us (6.8 TB/s).
//
// Rows start at any element: a row's vectors are the 16-byte blocks of its address, the
// full ones copied in bulk, a partial first or last one filled in by the producer's
// lanes with -infinity outside the row. Where logits and gradient rows are not aligned
// alike (mod 16 bytes) a gradient's vector is put together from two of the ring's.
//
// Every wait is bounded, between the warps too: one that expires ends the CTA's work and
// is reported as MALIB_ETIMEOUT.
#pragma once

#include "token_common.cuh"
#include "token_emit.cuh"
#include "token_peer.cuh"
#include "token_top.cuh"

namespace malib {

namespace {

// Consumer threads, vectors of each in a stage, CTAs an SM; what a thread gathers a row's
// statistics in.
struct RingSmall {
    static constexpr int kConsumers = 128, kPer = 8, kCtas = 3;
    using Own = RowStat;
};
struct RingStat {                                    // nothing is written
    static constexpr int kConsumers = 128, kPer = 8, kCtas = 4;
    using Own = RowStat;
};
struct RingLarge {
    static constexpr int kConsumers = 256, kPer = 8, kCtas = 2;
    using Own = RowStat;
};
struct RingHuge {
    static constexpr int kConsumers = 256, kPer = 8, kCtas = 1;
    using Own = RowStat;
};
// Slices of more than kManyParts stages. Kept for all lengths the errors of the additions cost 0.7 %
// of a policy loss of 16,384 x 131,072 and 2 % of log-probabilities of 8,192 x 20,000 (bf16).
constexpr int kManyParts = 16;
struct RingStatLong : RingStat {
    using Own = LongStat;
};
struct RingHugeLong : RingHuge {
    using Own = LongStat;
};
constexpr int kMaxStages = 6, kMaxCluster = 8;
constexpr int kQueue = 4;                            // most rows known ahead
constexpr int kRingMost = 216 * 1024;                // dynamic shared memory

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
    int32_t kind;                                    // kOutZero: no gradient; kOutSteep: an infinite slope
};
enum : int { kOutZero = 0, kOutPlain = 1, kOutSteep = 2 };

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
    int dealt;                                       // row t of CTA, or cluster, i is i + t times their number
    int l2;                                          // copies say how long the L2 cache should keep a part
};

// How long the L2 cache should keep what a copy reads.
__device__ __forceinline__ uint64_t l2_evict_first() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ uint64_t l2_evict_last() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void bulk_g2s_l2(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
            smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}

// The statistics of a call from its rows' shares, in the rows' order (every thread of one
// block).
template <int kOp, int kThreads>
__device__ __forceinline__ void sum_rows(const TokenArgs& a) {
    Totals v{};
    constexpr int kAt = 16;                          // loads in flight
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

template <class T, int kOp, class Ring>
__global__ void __launch_bounds__(Ring::kConsumers + (kOp == kTokDistill ? 64 : 32), Ring::kCtas)
    token_ring_kernel(TokenArgs a, Shape sh) {
    constexpr int W = Elt<T>::W;
    constexpr int kConsumers = Ring::kConsumers, kConsumerWarps = kConsumers / 32, kPer = Ring::kPer;
    constexpr int kStageVecs = kConsumers * kPer, kStageBytes = kStageVecs * 16;
    constexpr int kThreads = kConsumers + (kOp == kTokDistill ? 64 : 32);
    constexpr bool kTop = kOp == kTokDistill;
    using Own = typename Ring::Own;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages];
    // per queued row: known, no longer needed; per row that is read: the warps' statistics
    // are there, the CTAs', the result, the written slice
    __shared__ __align__(8) uint64_t qfull[kQueue], qempty[kQueue], sfull[kQueue], rfull[kQueue], pfull[kQueue],
        xfull[2];
    __shared__ __align__(8) uint64_t tfull[2], tempty[2];
    __shared__ Queued queue[kQueue];
    __shared__ Partial red[kQueue][kConsumerWarps], xslot[2][kMaxCluster];
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
        for (int i = 0; i < 2; ++i) {
            mbar_init(&xfull[i], 1);
            mbar_init(&tfull[i], 1);
            mbar_init(&tempty[i], kConsumerWarps);
        }
        fence_proxy_async_smem();
    }
    __syncthreads();
    wait_for_previous();
    if (kOp == kTokLogp) let_next_start();
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
    // Turn t's row, as every warp sees it; row < 0: there is none. A dealt row's token and
    // weight are asked for a turn ahead.
    Queued ahead{-1, -1, 0.f};
    if (sh.dealt && blockIdx.x / C < a.n) ahead = look(blockIdx.x / C);
    auto take = [&](uint32_t t) {
        Queued q{-1, -1, 0.f};
        if (sh.dealt) {
            q = ahead;
            ahead.row = -1;
            const int64_t next = q.row + gridDim.x / C;
            if (q.row >= 0 && next < a.n) ahead = look(next);
            settle(q, rank == 0 && tid == 0);
            return q;
        }
        wait(&qfull[slot_of(t)], parity_of(t));
        if (!*gone) q = queue[slot_of(t)];
        return q;
    };
    // The warp needs nothing of turn t any more.
    auto leave = [&](uint32_t t) {
        if (sh.dealt) return;
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
        if (!sh.dealt) look_batch();
        const uint64_t l2_first = l2_evict_first(), l2_last = l2_evict_last();
        Cursor at, issued;
        bool wrapped = false;
        for (uint32_t t = 0;; ++t) {
            if (!sh.dealt) {
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
                    if (fill) {
                        reinterpret_cast<T*>(dst)[(pv - v) * W + (lane & 15)] = entry;
                        fence_proxy_async_smem();    // a later use's copy overwrites what is stored here
                    }
                    __syncwarp();
                    if (*gone) break;
                    wrapped |= stage + 1 == sh.stages;
                    issued = at;
                    if (lane == 0) {
                        const int b0 = head ? 1 : 0, b1 = tail ? n - 1 : n;
                        const uint32_t bytes = b1 > b0 ? (uint32_t)(b1 - b0) * 16u : 0u;
                        mbar_arrive_expect_tx(&full[stage], bytes);
                        const T* src = z + ((int64_t)(v + b0) * W - h);
                        if (kOp != kTokLogp && bytes && sh.l2)
                            bulk_g2s_l2(dst + b0 * 16, src, bytes, &full[stage], part < again ? l2_last : l2_first);
                        else if (bytes)
                            bulk_g2s(dst + b0 * 16, src, bytes, &full[stage]);
                    }
                    __syncwarp();
                }
            }
            if (!sh.dealt && used == sh.batch) {
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
                    const TopRow r = top_row<T, kSeen>(a, q.row, static_cast<const T*>(a.z) + q.row * a.ld,
                                                       entries + b * a.top, seen);
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
                if (g) zero_entries<T, kConsumers>(tid, g, max(0, v_lo * W - h), max(0, min(a.V, v_hi * W - h)));
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
            Own own{};
            own.m = -INFINITY;
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
                raise(own, vec_max<T>(x), a.k);
                if (own.m != -INFINITY) gather<T>(own, x, a.k);
                if (part < kept) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(&empty[at.stage]);
                }
            }
            RowStat r = reduce_stat<32>(stat_of(own), a.k);
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
                    // before any CTA of the row writes its part: they go before these sums. Two
                    // rows' sums have places: a CTA sends the second next row's after it has
                    // the next one's of every peer, which sent them after reading this row's.
                    join();
                    if (lane == 0) mbar_arrive_expect_tx(&xfull[b], (uint32_t)(C * sizeof(Partial)));
                    if (lane < C) peer_store(&xslot[b][rank], &xfull[b], lane, make_float4(r.m, r.s, r.t, zt));
                    if (!*gone && !peer_wait_bounded(&xfull[b], turn >> 1 & 1u, kWaitLimitNs)) expired();
                    const Partial& px = xslot[b][lane & (kMaxCluster - 1)];
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
                        rout[slot] = RowOut{c, !live ? kOutZero : kOp == kTokPpo && is_steep(c) ? kOutSteep : kOutPlain};
                        mbar_arrive_release(&rfull[slot]);
                    }
                }
            }
            if (g) {
                wait(&rfull[slot], parity);
                const RowGrad c = rout[slot].c;
                const int kind = rout[slot].kind;
                const bool alike = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
                if (kept < parts) at = begin;
                for (int i = 0; i < parts; ++i, at.next(sh.stages)) {
                    const int part = kept + i < parts ? kept + i : kept + i - parts, v = v_lo + part * kStageVecs;
                    const int n = min(kStageVecs, v_hi - v), j = v * W - h;
                    if (part < kept) wait(&full[at.stage], at.parity);
                    const int j0 = max(0, j), j1 = min(a.V, j + n * W);
                    const uint8_t* src = ring + at.stage * kStageBytes;
                    const int token = kTop ? -1 : q.token;
                    if (kind != kOutPlain) {
                        if (kOp == kTokPpo && kind == kOutSteep)
                            emit_steep_part<T, kConsumers>(tid, reinterpret_cast<const T*>(src) - j, j0, j1, g, c, a.k, token);
                        else
                            zero_entries<T, kConsumers>(tid, g, j0, j1);
                    } else if (kOp == kTokPpo && c.c1 != 0.f)
                        emit_stage<T, true, kConsumers, kPer>(tid, src, j, j0, j1, n, g, alike, c, a.k, token);
                    else
                        emit_stage<T, false, kConsumers, kPer>(tid, src, j, j0, j1, n, g, alike, c, a.k, token);
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(&empty[at.stage]);
                }
                if (kTop) {
                    // the teacher's entries of this slice, over what the CTA's warps have written
                    if (lane == 0) mbar_arrive_release(&pfull[slot]);
                    wait(&pfull[slot], parity);
                    const int j0 = max(0, v_lo * W - h), j1 = min(a.V, v_hi * W - h);
                    if (kind == kOutPlain)
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
    if (!stats && sh.dealt) return;
    if (!last_of(a.ticket, gridDim.x)) return;
    if (tid == 0) *a.claims = 0ull;
    if (stats) sum_rows<kOp, kThreads>(a);
}

// `units` CTAs, or clusters; 0: as many clusters as the device holds, at most one a row.
template <class T, int kOp, class Ring>
cudaError_t launch_ring(const TokenArgs& a, const Shape& sh, int64_t units, cudaStream_t s) {
    cudaError_t e =
        cudaFuncSetAttribute(token_ring_kernel<T, kOp, Ring>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingMost);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[2] = {};
    cfg.gridDim = dim3((unsigned)((units ? units : 1) * sh.cluster));
    cfg.blockDim = dim3(Ring::kConsumers + (kOp == kTokDistill ? 64 : 32));
    cfg.dynamicSmemBytes = (size_t)sh.stages * Ring::kConsumers * Ring::kPer * 16 +
                           (kOp == kTokDistill ? 2 * a.top * sizeof(TopEntry) : 0);
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
    if (units == 0) {
        int most = 0;
        e = cudaOccupancyMaxActiveClusters(&most, token_ring_kernel<T, kOp, Ring>, &cfg);
        if (e != cudaSuccess) return e;
        cfg.gridDim.x = (unsigned)(most < 1 ? 1 : most < a.n ? most : a.n) * sh.cluster;
    }
    return cudaLaunchKernelEx(&cfg, token_ring_kernel<T, kOp, Ring>, a, sh);
}

template <class T, int kOp>
cudaError_t launch_ring_op(const TokenArgs& a, int n_sm, cudaStream_t s) {
    const int64_t nv = (a.V + 2 * (int64_t)Elt<T>::W - 2) / Elt<T>::W;               // most vectors of a row
    const bool write = kOp != kTokLogp && a.g != nullptr;
    auto slice = [&](int c) { return (nv + c - 1) / c; };
    // CTAs an SM by the bytes of a slice (the figures above): three of the small shape with
    // four stages, four with three where nothing is written; two or one of the large one
    // with three or six.
    auto ctas = [&](int c) { return !write ? 4 : slice(c) <= 7168 ? 3 : slice(c) <= 13312 ? 2 : 1; };
    // CTAs a row: as many as the device holds for all the rows at once, with slices of 8 KB
    // or more. Over more rounds than one the exchange costs what the finer share gains. In
    // us, C = 1, 2, 4 and 8, ppo bf16: 25 rows of 64 KB 13.1, 11.8, 11.9, 11.4; 120 13.2,
    // 13.0, 18.7, 21.7; 300 14.5, 22.9, 28.9, 43.5; 60 rows of 256 KB 20.8, 16.7, 15.8, 22.1.
    Shape sh{};
    sh.cluster = 1;
    for (int c = 2; c <= kMaxCluster && slice(c) >= 512; c *= 2)
        if (a.n * c <= (int64_t)ctas(c) * n_sm) sh.cluster = c;
    // Rows of 480 KB or more, over several rounds: slices of 240 KB or more, by clusters of 2
    // or 4 one row after another. Less of a row has to come again from the L2 cache, the
    // last round is shorter, and a slice of this length hides the exchange. us, C = 1, 2 and
    // 4: 333 rows of 604 KB 99, 91, 92; 1,200 of them 300, 252, 277; 200 rows of 500 KB 63,
    // 54, 56; 800 of 1 MB 341, 340, 301; 800 of 400 KB 126, 137, 163; 1,200 of 256 KB 114,
    // 139, 186.
    const bool again = write && sh.cluster == 1 && a.n > n_sm && slice(2) >= 15000;
    if (again) sh.cluster = slice(4) >= 15000 ? 4 : 2;
    const int per_sm = ctas(sh.cluster);
    const int64_t held = (int64_t)per_sm * n_sm;
    const int stage = (per_sm < 3 ? RingLarge::kConsumers : RingSmall::kConsumers) * RingSmall::kPer;
    sh.stages = per_sm == 4 ? 3 : per_sm == 3 ? 4 : per_sm == 2 ? 3 : 6;
    sh.slice = (int)slice(sh.cluster);
    sh.keep = sh.slice <= (sh.stages - 1) * stage ? sh.stages - 1 : sh.stages - 2;
    // Every row at once, or CTAs that claim rows, or clusters that they are dealt to.
    sh.dealt = sh.cluster > 1 || a.n <= held;
    const int64_t units = again ? 0 : sh.dealt ? a.n : held;
    // Rows of which the CTAs on the device hold some 45 MB or more between their sweeps: the
    // parts that come again are to stay in the L2 cache, the others and the second copies to
    // go. us without and with this: 1,111 rows of 200 KB (two CTAs an SM) 91.7 and 87.7,
    // 800 of 400 KB 126 and 120, 1,200 of 604 KB (clusters of 2) 252 and 246; rows of 256 KB
    // 329 and 332, of 100 KB no difference.
    sh.l2 = write && per_sm < 3 && per_sm * sh.slice >= 18000;
    // Rows of a stage or more are claimed one by one and known one ahead, so that no CTA holds
    // several while others run out; short ones in batches of about two stages, as long as
    // there are several for every CTA.
    sh.queue_log = sh.slice >= stage ? 1 : 2;
    sh.batch = 1;
    if (sh.slice < stage && !sh.dealt) {
        const int64_t most = a.n / (4 * held), about = 2 * stage / sh.slice;
        sh.batch = (int)(most < 1 ? 1 : most < about ? most : about);
        if (sh.batch > 16) sh.batch = 16;
    }
    const bool many = sh.slice > kManyParts * stage;
    if (per_sm == 4) return many ? launch_ring<T, kOp, RingStatLong>(a, sh, units, s) : launch_ring<T, kOp, RingStat>(a, sh, units, s);
    if constexpr (kOp != kTokLogp) {
        // (three or two CTAs an SM have slices of at most 7 stages)
        if (per_sm == 3) return launch_ring<T, kOp, RingSmall>(a, sh, units, s);
        if (per_sm == 2) return launch_ring<T, kOp, RingLarge>(a, sh, units, s);
        return many ? launch_ring<T, kOp, RingHugeLong>(a, sh, units, s) : launch_ring<T, kOp, RingHuge>(a, sh, units, s);
    }
    return cudaErrorInvalidValue;                    // (not reached)
}

template <class T>
cudaError_t launch_ring_type(const TokenArgs& a, int op, int n_sm, cudaStream_t s) {
    if (op == kTokLogp) return launch_ring_op<T, kTokLogp>(a, n_sm, s);
    if (op == kTokPpo) return launch_ring_op<T, kTokPpo>(a, n_sm, s);
    return launch_ring_op<T, kTokDistill>(a, n_sm, s);
}

}  // namespace

}  // namespace malib
