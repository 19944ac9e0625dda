// Shared by the mixture-of-experts kernels: element types, loads without an
// alignment, and the search for a workgroup's rows in the experts' offsets.
#pragma once

#include <hip/hip_runtime.h>
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

// Blocks of at most `rows` rows of one expert: at most this many.
inline int64_t row_blocks_bound(int64_t R, int64_t E, int64_t rows) {
    return R / rows + (E + 1 < R ? E + 1 : R);
}

// A workgroup's block of rows and its column tile.
struct RowTile {
    int e;                 // expert; -1: there is no such tile; E: rows of no expert
    int64_t first, end;    // the block's rows
    int col;               // column tile, 0 <= col < cols
};

// Tile `id` of an order that walks the experts, in each the column tiles, and
// in each of those the expert's row blocks: neighbours share the columns of one
// expert's matrix.  With xcd the workgroup number is first remapped (workgroup i
// runs on XCD i % 8) so that each XCD takes a contiguous run of tiles.  Called
// by all 64 lanes of a wave with the same arguments.
__device__ inline RowTile find_row_tile(const int *__restrict__ offsets, int E, int64_t R, int rows,
                                        int cols, int64_t id, bool xcd) {
    const int lane = threadIdx.x & 63;
    auto blocks_of = [&](int e) -> int64_t {
        if (e > E) return 0;
        int64_t lo, hi;
        expert_rows(offsets, E, R, e, lo, hi);
        return (hi - lo + rows - 1) / rows;
    };
    auto inclusive = [&](int64_t v) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t up = __shfl_up(v, d);
            if (lane >= d) v += up;
        }
        return v;
    };
    if (xcd) {
        int64_t total = 0;
        for (int e0 = 0; e0 <= E; e0 += 64) total += __shfl(inclusive(blocks_of(e0 + lane)), 63);
        total *= cols;
        const int64_t per = (total + 7) / 8;
        if (id / 8 >= per) return {-1, 0, 0, 0};
        id = id % 8 * per + id / 8;
        if (id >= total) return {-1, 0, 0, 0};
    }
    int64_t before = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const int64_t n = blocks_of(e0 + lane), upto = inclusive(n);
        const unsigned long long past = __ballot(id < (before + upto) * cols);
        if (past != 0) {
            const int at = __ffsll(past) - 1;
            const int64_t n_e = __shfl(n, at), start = before + __shfl(upto, at) - n_e;
            const int64_t r = id - start * cols;
            int64_t lo, hi;
            expert_rows(offsets, E, R, e0 + at, lo, hi);
            const int64_t first = lo + r % n_e * rows;
            return {e0 + at, first, first + rows < hi ? first + rows : hi, (int)(r / n_e)};
        }
        before += __shfl(upto, 63);
    }
    return {-1, 0, 0, 0};
}

}  // namespace emu
