// Products of 8-bit integers with many rows of each expert: the stream of k-blocks of
// grouped16.h on v_mfma 32 x 32 x 32 of 8-bit integers, a k-block of 128 indices (128
// bytes of a row, as there), sums in 32-bit integers (exact: at most 131071 products of
// at most 2^14).  Rows, and so K, are multiples of 16 bytes.
//
// K need not be whole k-blocks: the copies of chunks past its end repeat the last one, and
// once a k-block that is not whole has landed, the chunks past the end of X's rows in LDS
// are overwritten with zeros (those of W may then hold anything; one barrier more for
// a tile).
//
// y = x's scale times w's scale times the sum, rounded three times in FP32 (the sum, two
// products), then to the type.  A column whose scale could take the product with the
// sum out of FP32's range goes through FP64.
#pragma once

#include "grouped16.h"

namespace emu {
namespace {

constexpr int KB_BYTES = BK * 2, KB_CHUNKS = KB_BYTES / 16;

// Rows of 8-bit integers whose k-blocks need not be whole.
template <int RB>
struct ByteSide : Side<RB, CONTIG> {
    using S = Side<RB, CONTIG>;
    int chunk[2], back[2];          // chunk of even and odd copies; how far it lies past the end, in bytes
    __device__ __forceinline__ void init_lane(int wave, int lane, int part) {
        S::init_lane(wave, lane, part);
#pragma unroll
        for (int c = 0; c < 2; ++c) chunk[c] = (lane % S::Q) ^ S::place(S::row_of(c, wave, lane));
    }
    // before the copies of k-block kb of rows of `chunks` chunks
    __device__ __forceinline__ void clamp(int kb, int chunks) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int past = kb * KB_CHUNKS + chunk[c] - (chunks - 1);
            back[c] = (past > 0 ? past : 0) << 4;
        }
    }
    // (the last chunk may lie before the k-block: its first address is taken, not an offset below 0)
    __device__ __forceinline__ void copy(int c, int kb, char *stage, int wave) const {
        copy_lanes(S::base, S::off[c] + (unsigned)(kb * KB_BYTES - back[c & 1]), stage + (wave * S::COPIES + c) * 1024);
    }
};

template <typename T, int RB, bool GATHER>
struct Q8Source {
    static constexpr int TILE = 64 * RB;
    using A = ByteSide<RB>;
    using B = ByteSide<RB>;
    static_assert(A::COPIES % 2 == 0, "a wave's copies start at an even one");
    const Q8Gemm &g;
    const TileList &list;
    int i;                          // list entry of `next`
    RowTile now, next;              // the tile that is computed, and the one after
    A a;
    B b;
    int kb, KB, chunks, wave, lane;
    int raw[A::COPIES], row[RB];    // look-ups: of the next tile's copies; X's rows of the rows to store, -1: none

    __device__ __forceinline__ Q8Source(const Q8Gemm &g_, const TileList &list_, int wave_, int lane_)
        : g(g_), list(list_), i(0), wave(wave_), lane(lane_) {
        a.init_lane(wave, lane, wave >> 1);
        b.init_lane(wave, lane, wave & 1);
        chunks = g.K / 16;
        KB = chunks <= 2 * KB_CHUNKS ? 2 : (chunks + KB_CHUNKS - 1) / KB_CHUNKS;
        now = next = list.at(0);
    }
    // whether the tile is a product (not one of the rows of no expert, the last ones)
    __device__ __forceinline__ bool product(const RowTile &t) const { return t.e >= 0 && t.e < g.E; }
    __device__ __forceinline__ void look_up() {
        if constexpr (GATHER) {
#pragma unroll
            for (int c = 0; c < A::COPIES; ++c) {
                const int r = (int)next.first + A::row_of(c, wave, lane);
                raw[c] = g.rows[r < next.end ? r : (int)next.end - 1];
            }
        }
    }
    // a and b for the tile `next`, from its look-ups; rows outside are read
    // from row 0 and zeroed where they are stored
    __device__ __forceinline__ void point() {
        const int rows = (int)(next.end - next.first), n0 = next.col * TILE;
        const int cols = g.N - n0 < TILE ? g.N - n0 : TILE;
        const int8_t *const W = g.W + next.e * g.sw + n0 * g.ldw;
        // leading dimensions in pairs
        a.init(reinterpret_cast<const char *>(g.X + (GATHER ? 0 : next.first * g.ldx)), g.ldx / 2, wave, lane,
               [&](int c, int r) -> unsigned {
                   if constexpr (!GATHER) return r < rows ? r : rows - 1;
                   return raw[c] >= 0 && raw[c] < g.xrows ? raw[c] : 0;
               });
        b.init(reinterpret_cast<const char *>(W), g.ldw / 2, wave, lane,
               [&](int, int r) -> unsigned { return r < cols ? r : cols - 1; });
        kb = 0;
    }
    __device__ __forceinline__ bool start() {
        if (!product(next)) return false;
        look_up();
        point();
        return true;
    }
    __device__ __forceinline__ void open() {
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const int64_t r = now.first + ((wave >> 1) * RB + j) * 32 + (lane & 31);
            row[j] = (int)(r < now.end ? r : now.end - 1);
            if (g.scaled) row[j] = g.scaled[row[j]];
        }
        // after the last product its own k-blocks are copied again, unused
        const RowTile t = list.at(i + 1);
        if (product(t)) next = t;
        ++i;
        look_up();
    }
    __device__ __forceinline__ void trip() {}
    // zeros past the end of X's rows
    __device__ __forceinline__ void arrived(char *stage, int block) {
        const int first = chunks - block * KB_CHUNKS;
        if (first >= KB_CHUNKS) return;
        const int r = threadIdx.x;
        if (r < A::ROWS)
            for (int q = first < 0 ? 0 : first; q < KB_CHUNKS; ++q)
                *reinterpret_cast<i32x4 *>(stage + r * A::RS + ((q ^ A::place(r)) << 4)) = i32x4{};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        pipeline_barrier();
    }
    __device__ __forceinline__ void landed() {
        if (kb == KB) point();
        a.clamp(kb, chunks);
        b.clamp(kb, chunks);
    }
    __device__ __forceinline__ void copied() { ++kb; }
    __device__ __forceinline__ int blocks() const { return KB; }
    __device__ __forceinline__ bool close(const i32x16 (&acc)[RB][RB]) {
        store(acc);
        now = next;
        return product(list.at(i));
    }
    // Register r of lane l is column 8 (r / 4) + 4 (l / 32) + r % 4 of row l % 32 of its
    // block.  16-bit results are exchanged between the lane halves: eight neighbouring
    // columns of a row to a lane, one 16-byte store.
    __device__ __forceinline__ void store(const i32x16 (&acc)[RB][RB]) const {
        const int n0 = now.col * TILE, cols = g.N - n0 < TILE ? g.N - n0 : TILE, h = lane >> 5;
        const float *const ws = g.ws + (int64_t)now.e * g.N + n0;
        T *const Y = static_cast<T *>(g.Y) + now.first * g.ldy + n0;
        const int rows = (int)(now.end - now.first);
        float xs[RB];
        bool there[RB];                                 // zeros for a row outside X, whatever W's scale
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            there[i] = row[i] >= 0 && row[i] < g.xrows;
            xs[i] = g.xs[there[i] ? row[i] : 0];
        }
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                const int col = ((wave & 1) * RB + j) * 32 + 2 * r;     // of 16 columns
                float w[8];
                bool wide = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int c = col + 8 * (k / 4) + 4 * h + k % 4;
                    w[k] = ws[c < cols ? c : cols - 1];
                    const float m = fabsf(w[k]);
                    wide |= m > 0x1p96f || (m < 0x1p-126f && m > 0.0f);
                }
                wide = __any(wide);
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    __builtin_amdgcn_sched_barrier(0);      // few values in flight: no registers to spare
                    float y[8];
                    if (wide) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = (float)((double)acc[i][j][r + k] * w[k] * xs[i]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = (float)acc[i][j][r + k] * w[k] * xs[i];
                    }
                    store8(Y, ((wave >> 1) * RB + i) * 32 + (lane & 31), rows, there[i], col, cols, y);
                }
            }
    }
    // y: columns 4 h .. 4 h + 3 and 8 + 4 h .. of the 16 from col on
    __device__ __forceinline__ void store8(T *Y, int row, int rows, bool keep, int col, int cols,
                                           const float (&y)[8]) const {
        const int h = lane >> 5;
        T *const p = Y + row * g.ldy;
        if constexpr (sizeof(T) == 4) {
            if (row >= rows) return;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int c = col + 8 * q + 4 * h;
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = keep ? y[4 * q + k] : 0.0f;
                if (c + 4 <= cols) {
                    store_f32<4>(p + c, v);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (c + k < cols) p[c + k] = v[k];
                }
            }
        } else {
            typedef T t2 __attribute__((ext_vector_type(2)));
            typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
            typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
            auto pack = [](float a, float b) {
                const t2 v = {(T)a, (T)b};
                return __builtin_bit_cast(unsigned, v);
            };
            const u32x2 u = __builtin_amdgcn_permlane32_swap(pack(y[0], y[1]), pack(y[4], y[5]), false, false);
            const u32x2 v = __builtin_amdgcn_permlane32_swap(pack(y[2], y[3]), pack(y[6], y[7]), false, false);
            u32x4 w = {u[0], v[0], u[1], v[1]};
            if (row >= rows) return;
            if (!keep) w = u32x4{};
            const int c = col + 8 * h;
            const frag<T> f = __builtin_bit_cast(frag<T>, w);
            if (c + 8 <= cols) {
                *reinterpret_cast<vec<T, 8> *>(p + c) = f;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) p[c + k] = f[k];
            }
        }
    }
};

template <typename T, int RB, bool GATHER>
__global__ __launch_bounds__(256, RB == 4 ? 1 : 2) void q8_tiles_kernel(Q8Gemm g) {
    using Source = Q8Source<T, RB, GATHER>;
    __shared__ __attribute__((aligned(1024))) char lds[2 * (Source::A::BYTES + Source::B::BYTES)];
    __shared__ TileList list;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    list.fill(g, Source::TILE);
    Source src(g, list, wave, lane);
    if (src.start()) run_tiles<i8pair, RB>(src, lds, wave);
    // rows of no expert
    for (int i = src.i; list.at(i).e == g.E; ++i) {
        const RowTile t = list.at(i);
        const int64_t n0 = (int64_t)t.col * Source::TILE;
        const int cols = (int)(g.N - n0 < Source::TILE ? g.N - n0 : Source::TILE);
        const int n = (int)(t.end - t.first) * cols;
        T *const C = static_cast<T *>(g.Y) + t.first * g.ldy + n0;
        for (int j = threadIdx.x; j < n; j += 256) C[j / cols * g.ldy + j % cols] = T(0.0f);
    }
}

template <typename T>
hipError_t launch_q8_tiles(const Q8Gemm &g, int tile, hipStream_t s) {
    auto run = [&](auto rb) {
        constexpr int RB = decltype(rb)::value, TILE = 64 * RB;
        const int64_t tiles = row_blocks_bound(g.R, g.E, TILE) * ((g.N + TILE - 1) / TILE);
        const unsigned grid = workgroups(tiles, RB == 4 ? 1 : 2);
        if (g.rows) q8_tiles_kernel<T, RB, true><<<grid, 256, 0, s>>>(g);
        else q8_tiles_kernel<T, RB, false><<<grid, 256, 0, s>>>(g);
    };
    if (tile == 256) run(std::integral_constant<int, 4>{});
    else run(std::integral_constant<int, 2>{});
    return hipGetLastError();
}

}  // namespace
}  // namespace emu
