// Shared by the mixture-of-experts kernels: element types, loads without an
// alignment, and the search for a workgroup's rows in the experts' offsets.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/emu.h"

namespace emu {

using half = _Float16;
using bhalf = __bf16;

// f(T{}) with the element type of an EMU_F32 / EMU_BF16 / EMU_F16 code.
template <typename F>
inline auto with_type(int dtype, F &&f) {
    if (dtype == EMU_F32) return f(float{});
    if (dtype == EMU_BF16) return f(bhalf{});
    return f(half{});
}
inline bool is_dtype(int dtype) { return dtype == EMU_F32 || dtype == EMU_BF16 || dtype == EMU_F16; }

// A vector of N elements that may start at any element: the hardware loads and
// stores 4 to 16 bytes at any address, at full speed where it is aligned.
template <typename T, int N>
using vec __attribute__((ext_vector_type(N), aligned(alignof(T)))) = T;

template <int N, typename T>
__device__ __forceinline__ void load_f32(const T *p, float (&x)[N]) {
    const vec<T, N> v = *reinterpret_cast<const vec<T, N> *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}
template <int N, typename T>
__device__ __forceinline__ void store_f32(T *p, const float (&x)[N]) {
    vec<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    *reinterpret_cast<vec<T, N> *>(p) = v;
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
// Sixteen bytes from k on of a row of K of them, zeros past its end: where that is inside of them,
// the row's last sixteen, moved down.
__device__ __forceinline__ i32x4 load_bytes16(const int8_t *row, int k, int K) {
    typedef int __attribute__((ext_vector_type(4), aligned(1))) unaligned;
    typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
    i32x4 v = {};
    if (K < 16) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (k + j < K) v[j / 4] |= (int)(uint8_t)row[k + j] << (8 * (j % 4));
        return v;
    }
    const int past = k + 16 - K;
    v = *reinterpret_cast<const unaligned *>(row + (past > 0 ? K - 16 : k));
    if (past <= 0) return v;
    u64x2 u = __builtin_bit_cast(u64x2, v);
    if (past >= 8) u = u64x2{u[1], 0};
    const int bits = 8 * (past & 7);
    u64x2 moved = {u[0] >> bits | (bits > 0 ? u[1] << (64 - bits) : 0), u[1] >> bits};
    if (past >= 16) moved = u64x2{};
    return __builtin_bit_cast(i32x4, moved);
}

// Rows of expert e: [lo, hi).  offsets (device, E + 1 entries; the first counts
// as 0) are clamped to [0, R], so that wrong ones cannot lead outside; e == E
// stands for the rows that belong to no expert, [offsets[E], R).  Without
// offsets all rows belong to expert 0.
__device__ inline void expert_rows(const int *__restrict__ offsets, int E, int64_t R, int e,
                                   int64_t &lo, int64_t &hi) {
    if (offsets == nullptr) {
        lo = e == 0 ? 0 : R;
        hi = R;
        return;
    }
    const int64_t a = e == 0 ? 0 : offsets[e], b = e == E ? R : offsets[e + 1];
    lo = a < 0 ? 0 : (a < R ? a : R);
    hi = b < lo ? lo : (b < R ? b : R);
}

// Piece i of `pieces` of an expert's rows: multiples of 64 rows, the last the rest.
__device__ inline void piece_rows(int i, int pieces, int64_t &lo, int64_t &hi) {
    const int64_t per = ((hi - lo + pieces - 1) / pieces + 63) & ~(int64_t)63, first = lo + i * per;
    lo = first < hi ? first : hi;
    hi = lo + per < hi ? lo + per : hi;
}

// The first of the tiles of XCD x (0 .. 8), where every expert has `each` tiles, one
// after the other, that take a time of its rows and START more: the XCDs get
// contiguous runs of tiles that take the same time.  By a whole wave; in all lanes.
__device__ inline int64_t first_tile_of_xcd(const int *__restrict__ offsets, int E, int64_t R, int64_t each, int x) {
    constexpr int START = 256;
    if (x == 8) return E * each;
    const int lane = threadIdx.x & 63;
    auto time_of = [&](int e) -> int64_t {
        if (e >= E) return 0;
        int64_t lo, hi;
        expert_rows(offsets, E, R, e, lo, hi);
        return hi - lo + START;
    };
    int64_t total = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        int64_t t = time_of(e0 + lane);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d);
        total += t;
    }
    int64_t target = total * x / 8;
    for (int e0 = 0;; e0 += 64) {
        const int64_t t = time_of(e0 + lane);
        int64_t upto = t;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t up = __shfl_up(upto, d);
            if (lane >= d) upto += up;
        }
        const uint64_t past = __ballot(upto > target);            // the expert: the first of these
        if (past == 0 && e0 + 64 < E) {
            target -= __shfl(upto, 63);
            continue;
        }
        const int at = past == 0 ? 63 : __ffsll((unsigned long long)past) - 1;
        const int64_t before = __shfl(upto - t, at), own = __shfl(t, at);
        const int64_t tile = (e0 + at) * each + (own > 0 ? (target - before) * each / own : 0);
        return tile < E * each ? tile : E * each;
    }
}

// Blocks of at most `rows` rows of one expert: at most this many.
inline int64_t row_blocks_bound(int64_t R, int64_t E, int64_t rows) {
    return R / rows + (E + 1 < R ? E + 1 : R);
}
// Experts that an even load of the rows reaches, and about so many blocks: an expert's
// last one is half full on average.
inline double experts_reached(int64_t R, int64_t E) { return E == 1 ? 1 : E * (1 - pow(1 - 1.0 / E, (double)R)); }
inline int64_t row_blocks_expected(int64_t R, int64_t E, int64_t rows) {
    if (E == 1) return (R + rows - 1) / rows;
    const double reached = experts_reached(R, E), blocks = (R + reached * rows / 2) / rows;
    return (int64_t)(blocks > reached ? blocks : reached + 0.5);
}

// A value that all lanes hold, below 2^31, in a scalar register.
__device__ __forceinline__ int uniform(int64_t v) { return __builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ const char *uniform(const char *p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v), hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
    return reinterpret_cast<const char *>((uint64_t)hi << 32 | lo);
}

// v summed over the lanes of the wave up to this one, in register moves between lanes
// (rows of 16 lanes, then the last lane of one or two rows to those behind).
__device__ __forceinline__ int sum_up_to_lane(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);     // row_shr 1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);     // row_shr 2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);     // row_shr 4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);     // row_shr 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     // row_bcast 15
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);     // row_bcast 31
    return v;
}

// v of another lane: within 16 lanes by moves between registers (0xB1, 0x4E: the lane's
// neighbour and the other pair of its four; 0x141, 0x140: its eight and its 16 mirrored).
template <int CTRL, typename T>
__device__ __forceinline__ T moved(T v) {
    return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

// f over LANES lanes (4, 16 or 64), in all of them; f is associative and commutative but
// for roundings, which are alike in every lane: f(a, b) and f(b, a) are.
template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f) {
    v = f(v, moved<0xB1>(v));
    v = f(v, moved<0x4E>(v));
    if constexpr (LANES > 4) {
        v = f(v, moved<0x141>(v));
        v = f(v, moved<0x140>(v));
    }
#pragma unroll
    for (int d = 16; d < LANES; d <<= 1) v = f(v, __shfl_xor(v, d));
    return v;
}

// exp(x - m) for x <= m; equal infinities give 1, -inf and NaN 0
__device__ __forceinline__ float exp_below(float x, float m) {
    return x == m ? 1.0f : (x > -INFINITY ? expf(x - m) : 0.0f);
}

// An 8-bit product's result from its sum and the scales of W's and X's row: three roundings in
// FP32, the same in every kernel, so that a row's bits do not depend on which one runs.  Where
// w could take its product with a sum (below 2^31) out of the range of normal numbers,
// mantissas are multiplied and exponents added.
__device__ __forceinline__ bool q8_extreme(float w) {
    const unsigned e = __float_as_uint(w) >> 23 & 255;
    return e > 222 || (e == 0 && w != 0.0f);        // 2^96 and more, not finite; subnormal
}
__device__ __forceinline__ float q8_result(int sum, float w, float x) {
    const bool parts = q8_extreme(w);
    const float mw = parts ? __builtin_amdgcn_frexp_mantf(w) : w, mx = parts ? __builtin_amdgcn_frexp_mantf(x) : x;
    return ldexpf((float)sum * mw * mx, parts ? __builtin_amdgcn_frexp_expf(w) + __builtin_amdgcn_frexp_expf(x) : 0);
}

// The operands and sums of the workgroup's split (see Q8Gemm::part).
template <typename Gemm>
__device__ __forceinline__ void to_split(Gemm &g) {
    const int i = blockIdx.y, first = i * g.part;
    g.X += first;
    g.W += first;
    g.K = g.K - first < g.part ? g.K - first : g.part;
    g.Y = static_cast<int *>(g.Y) + i * g.R * g.ldy;
}

// A workgroup's block of rows and its column tile.
struct RowTile {
    int e;                 // expert; -1: there is no such tile; E: rows of no expert
    int64_t first, end;    // the block's rows
    int col;               // column tile, 0 <= col < cols
};

// The row tiles of a product, in an order that walks the experts, in each groups
// of eight row blocks, in each of those the column tiles, then the row blocks:
// the tiles that run at a time share few rows and few columns of one expert.
// Used by all 64 lanes of a wave with the same arguments; the first 64 experts'
// blocks are counted once.
struct RowTiles {
    const int *offsets;
    int E, rows, cols;
    int64_t R;
    int n0, upto0;                  // blocks of expert `lane`, and of those up to it
    int64_t total;                  // tiles

    __device__ __forceinline__ int blocks_of(int e) const {
        if (e > E) return 0;
        int64_t lo, hi;
        expert_rows(offsets, E, R, e, lo, hi);
        return (int)(((unsigned)(hi - lo) + rows - 1) / rows);
    }
    __device__ __forceinline__ RowTiles(const int *offsets_, int E_, int64_t R_, int rows_, int cols_)
        : offsets(offsets_), E(E_), rows(rows_), cols(cols_), R(R_) {
        const int lane = threadIdx.x & 63;
        n0 = blocks_of(lane);
        upto0 = sum_up_to_lane(n0);
        total = __builtin_amdgcn_readlane(upto0, 63);
        for (int e0 = 64; e0 <= E; e0 += 64)
            total += __builtin_amdgcn_readlane(sum_up_to_lane(blocks_of(e0 + lane)), 63);
        total *= cols;
    }
    // the tile of workgroup w: workgroup w runs on XCD w % 8, and an XCD takes a
    // contiguous run of tiles
    __device__ __forceinline__ RowTile of_workgroup(int64_t w) const {
        const int64_t per = (total + 7) / 8, id = w % 8 * per + w / 8;
        if (w / 8 >= per || id >= total) return {-1, 0, 0, 0};
        return at(id);
    }
    __device__ __forceinline__ RowTile at(int64_t id) const {
        const RowTile t = search(id);
        return {uniform(t.e), uniform(t.first), uniform(t.end), uniform(t.col)};
    }
    __device__ inline RowTile search(int64_t id) const {
        const int lane = threadIdx.x & 63;
        int n = n0, upto = upto0;
        int64_t before = 0;
        for (int e0 = 0;;) {
            const unsigned long long past = __ballot(id < (before + upto) * cols);
            if (past != 0) {
                const int i = __ffsll(past) - 1;
                const int n_e = __builtin_amdgcn_readlane(n, i);
                const int64_t start = before + __builtin_amdgcn_readlane(upto, i) - n_e;
                const int r = (int)(id - start * cols);
                int64_t lo, hi;
                expert_rows(offsets, E, R, e0 + i, lo, hi);
                const int g0 = r / (8 * cols) * 8, in = r - g0 * cols;
                const int high = n_e - g0 < 8 ? n_e - g0 : 8;
                const int64_t first = lo + (int64_t)(g0 + in % high) * rows;
                return {e0 + i, first, first + rows < hi ? first + rows : hi, in / high};
            }
            before += __builtin_amdgcn_readlane(upto, 63);
            e0 += 64;
            if (e0 > E) return {-1, 0, 0, 0};
            n = blocks_of(e0 + lane);
            upto = sum_up_to_lane(n);
        }
    }
};

// One 1 KB copy: lane l moves 16 bytes from its own source to dst + 16 l (dst
// and base uniform over the wave).  Inline asm, which has no output register:
// the compiler takes a transposing LDS read to depend on every such copy in
// flight and would wait for the one just issued before each read.  The kernels
// wait for them themselves (s_waitcnt vmcnt before a barrier).  The s_nop is
// the wait state between a write of m0 (which the compiler keeps nothing in) and
// its use by the copy.
__device__ __forceinline__ unsigned lds_address(char *p) {
    return (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)p;
}
__device__ __forceinline__ void copy_lanes(const char *base, unsigned offset, char *dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds_address(dst)), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void copy_lanes(const char *src, char *dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(lds_address(dst)), "v"(src) : "memory");
}
// The same for 4 bytes of a lane: to dst + 4 l.
__device__ __forceinline__ void copy_lanes4(const void *src, char *dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 :: "s"(lds_address(dst)), "v"(src) : "memory");
}

}  // namespace emu
