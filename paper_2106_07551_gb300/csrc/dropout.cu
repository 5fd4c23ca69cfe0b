// Dropout whose mask is a function of its place: element (row, column) is kept by 16 bits of
// Philox4x32-10 at counter (sequence, step, 2^31 | site << 16 | column / 8), so that no mask is
// stored and a batch put together in another order sees the same one.
//   out = residual + (bits >= p 2^16 ? x / (1 - p) : 0)
// in fp32 with one rounding, then the one to the type. A call of the generator has 128 bits: eight
// columns, of word i the low half for column 2 i, the high half for 2 i + 1.
//
// A thread writes eight columns that start on a 16-byte boundary of out. Where rows start inside
// such a vector it spans two calls of the generator; a lane has one of them and takes the other's bits
// from the lane before, so that 31 lanes of a warp write. x and residual that are not aligned as
// out is are put together from two vectors.
//
// Memory bounds it, then the generator's multiplications: 32,768 x 8,192 bf16 with a residual 278 us (5.8 TB/s
// of the measured 6.8; ALU pipe 58 %, issue slots 62 %), 102,400 x 64 fp32 11.2 us (4.8 TB/s). A
// mask in memory would be a bit an element more to read and write, and could not be had again.
#include "token_rollout.h"
#include "token_shift.cuh"

namespace malib {

namespace {

constexpr int kDropThreads = 256;

// Bit e: column 8 block + e is kept.
__device__ __forceinline__ uint32_t keep_bits(const DropArgs& a, uint64_t sequence, uint32_t step, uint32_t block) {
    const U4 w = draw(sequence, step, a.counter | block, a.seed);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        bits |= ((v[i] & 0xffffu) >= a.least ? 1u << 2 * i : 0u) | (v[i] >> 16 >= a.least ? 2u << 2 * i : 0u);
    return bits;
}

// Columns j .. j + 7 of a row, 0 outside [0, d).
template <class T>
struct Eight {
    static constexpr int W = Elt<T>::W, N = 8 / W;
    uint4 q[N];
    __device__ __forceinline__ void load(const T* row, int j, int d) {
        if (j >= 0 && j + 8 <= d) {
            const T* p = row + j;
            const int by = (int)((uintptr_t)p & 15u);
            if (by == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) q[i] = reinterpret_cast<const uint4*>(p)[i];
                return;
            }
            const int first = j - by / (int)sizeof(T);               // of the vectors that hold them
            if (first >= 0 && first + 8 + W <= d) {
#pragma unroll
                for (int i = 0; i < N; ++i) q[i] = load_shifted(reinterpret_cast<const uint8_t*>(p) - by + 16 * i, by);
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            F2 v[W / 2];
#pragma unroll
            for (int e = 0; e < W; e += 2) {
                const int c = j + i * W + e;
                v[e / 2] = f2_make(c >= 0 && c < d ? Elt<T>::get(row[c]) : 0.f, c + 1 >= 0 && c + 1 < d ? Elt<T>::get(row[c + 1]) : 0.f);
            }
            q[i] = Elt<T>::pack(v);
        }
    }
};

template <class T, bool kAligned, bool kResidual>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(DropArgs a) {
    constexpr int W = Elt<T>::W, N = 8 / W, kWarps = kDropThreads / 32, kOwn = kAligned ? 32 : 31;
    constexpr int kTile = kWarps * kOwn;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = a.per_row;                       // vectors of a row
    wait_for_previous();
    let_next_start();
    // the tile's first vector is i0 of row r0; the next tile of this block is (step_r, step_i) on
    int64_t r0 = (int64_t)blockIdx.x * kTile / per;
    int i0 = (int)((int64_t)blockIdx.x * kTile - r0 * per);
    for (; r0 < a.n; r0 += a.step_r, i0 += a.step_i) {
        if (i0 >= per) {
            i0 -= per;
            if (++r0 >= a.n) break;
        }
        // vector `at` of the tile: lane 0 of a warp whose lanes share bits has the one before its first
        const int at = warp * kOwn + lane - (kAligned ? 0 : 1);
        int i = i0 + at;
        int64_t row = r0;
        if (i < 0) {
            row -= 1;
            i += per;
        }
        if (i >= per) {
            const int q = per >= kTile ? 1 : per == 1 ? i : (int)__umulhi((uint32_t)i, a.magic);
            row += q;
            i -= q * per;
        }
        const bool inside = row >= 0 && row < a.n;
        uint32_t bits = 0;
        T* out = nullptr;
        int j = 0;
        Eight<T> x, res;
        const bool mine = inside && (kAligned || lane > 0);
        if (inside) {
            out = static_cast<T*>(a.out) + row * a.ld_out;
            j = 8 * i;
            if (!kAligned) j -= (int)(((uintptr_t)out & 15u) / sizeof(T));
            if (mine && j < a.d) {
                x.load(static_cast<const T*>(a.x) + row * a.ld_x, j, a.d);
                if (kResidual) res.load(static_cast<const T*>(a.residual) + row * a.ld_res, j, a.d);
            }
            bits = keep_bits(a, (uint64_t)a.sequence[row], (uint32_t)a.step[row], (uint32_t)i);
        }
        if (!kAligned) {
            const uint32_t before = __shfl_up_sync(0xffffffffu, bits, 1);
            bits = (before | bits << 8) >> (8 - (8 * i - j));
        }
        if (!mine || j >= a.d) continue;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            F2 v[W / 2], r[W / 2];
            Elt<T>::pairs(x.q[n], v);
            if (kResidual) Elt<T>::pairs(res.q[n], r);
#pragma unroll
            for (int e = 0; e < W / 2; ++e) {
                const float2 f = f2_split(v[e]), g = kResidual ? f2_split(r[e]) : make_float2(0.f, 0.f);
                const uint32_t b = bits >> (n * W + 2 * e);
                v[e] = f2_make(b & 1u ? fmaf(f.x, a.scale, g.x) : g.x, b & 2u ? fmaf(f.y, a.scale, g.y) : g.y);
            }
            const uint4 y = Elt<T>::pack(v);
            const int c = j + n * W;
            if (c >= 0 && c + W <= a.d) *reinterpret_cast<uint4*>(out + c) = y;
            else store_part(out + c, c, a.d, y);
        }
    }
}

template <class T, bool kAligned>
cudaError_t launch_dropout_as(DropArgs a, int n_sm, cudaStream_t s) {
    constexpr int kTile = kDropThreads / 32 * (kAligned ? 32 : 31);
    a.per_row = (a.d + (kAligned ? 0 : Elt<T>::W - 1) + 7) / 8;
    const int64_t tiles = a.n <= INT64_MAX / a.per_row ? (a.n * a.per_row + kTile - 1) / kTile : INT64_MAX;
    const int64_t grid = tiles < 8 * (int64_t)n_sm ? tiles : 8 * (int64_t)n_sm;
    a.step_r = grid * kTile / a.per_row;
    a.step_i = (int)(grid * kTile % a.per_row);
    a.magic = a.per_row > 1 ? (uint32_t)(((1ull << 32) + a.per_row - 1) / a.per_row) : 0;
    return a.residual ? launch_after(dropout_kernel<T, kAligned, true>, (unsigned)grid, kDropThreads, 0, s, a)
                      : launch_after(dropout_kernel<T, kAligned, false>, (unsigned)grid, kDropThreads, 0, s, a);
}
template <class T>
cudaError_t launch_dropout_type(const DropArgs& a, int n_sm, cudaStream_t s) {
    const bool aligned = ((uintptr_t)a.out & 15u) == 0 && (a.n == 1 || a.ld_out % Elt<T>::W == 0);
    return aligned ? launch_dropout_as<T, true>(a, n_sm, s) : launch_dropout_as<T, false>(a, n_sm, s);
}

}  // namespace

cudaError_t launch_dropout(const DropArgs& a, int n_sm, cudaStream_t s) {
    if (a.dtype == MALIB_F32) return launch_dropout_type<float>(a, n_sm, s);
    if (a.dtype == MALIB_BF16) return launch_dropout_type<__nv_bfloat16>(a, n_sm, s);
    return launch_dropout_type<__half>(a, n_sm, s);
}

}  // namespace malib
