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
// Results as q8_result forms them.  Tiles whose columns and rows of X all exist, and none of
// whose scales is extreme, are stored without checks (131072 rows below: 336 -> 309 us).
//
// Tiles of 256 hold one workgroup to a CU; of tiles of 128, a quarter of the accumulators each,
// two share one, or one has four stages, three k-blocks of copies in flight, where there are no
// more tiles than CUs.  Those read fragments two sub-steps ahead: a sub-step of theirs is four
// MFMAs long, less than the latency of an LDS read under load.
//
// Measured in bfloat16: 8192 x 8192 x 8192 439 to 466 us (2.4 to 2.5 POP/s, MFMA busy for 64 % of the
// cycles at 1.8 GHz, the power limit); 131072 gathered rows over 64 experts of 1024 x 2048 295 to
// 308 us, of which forming the results is 28 and storing them 34.  A k-block of a tile of 128
// takes 0.45 us (1000 cycles) however few run, its MFMAs 512 cycles: the LDS takes 32 KB of
// copies (as if at 64 bytes a cycle) and gives 64 KB of fragments.
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
    // (the last chunk may lie before the k-block: the sum is its offset in the row all the same)
    __device__ __forceinline__ void copy(int c, int kb, char *stage, int wave) const {
        copy_lanes(S::base, S::off[c] + (unsigned)(kb * KB_BYTES - back[c & 1]), stage + (wave * S::COPIES + c) * 1024);
    }
};

// The scales of a tile's rows and columns, and which rows exist in X.
template <int TILE>
struct Scales {
    float x[TILE], w[TILE];
    int there[TILE];
};

template <typename T, int RB, int STAGES, bool GATHER>
struct Q8Source {
    static constexpr int TILE = 64 * RB;
    static constexpr bool SUMS = std::is_same<T, int>::value;   // 32-bit sums without scales
    using Out = std::conditional_t<SUMS, float, T>;             // their bits
    using A = ByteSide<RB>;
    using B = ByteSide<RB>;
    static_assert(A::COPIES % 2 == 0, "a wave's copies start at an even one");
    const Q8Gemm &g;
    const TileList &list;
    Scales<TILE> (&scales)[2];      // of the tile and the one after, in turn
    int i;                          // list entry of `next`
    RowTile now, next;              // the tile that is computed, and the one after
    A a;
    B b;
    int kb, KB, chunks, wave, lane;
    int raw[A::COPIES];             // look-ups of the next tile's copies
    int row, turn;                  // X's row of row threadIdx.x of the tile that is computed next; 0 or 1

    __device__ __forceinline__ Q8Source(const Q8Gemm &g_, const TileList &list_, Scales<TILE> (&scales_)[2], int wave_,
                                        int lane_)
        : g(g_), list(list_), scales(scales_), i(0), wave(wave_), lane(lane_), turn(1) {
        a.init_lane(wave, lane, wave >> 1);
        b.init_lane(wave, lane, wave & 1);
        chunks = g.K / 16;
        KB = chunks <= STAGES * KB_CHUNKS ? STAGES : (chunks + KB_CHUNKS - 1) / KB_CHUNKS;
        now = next = list.at(0);
    }
    // whether the tile is a product (not one of the rows of no expert, the last ones)
    __device__ __forceinline__ bool product(const RowTile &t) const { return t.e >= 0 && t.e < g.E; }
    // the lane, so that what is made from it is made where it is needed, not kept through the tiles
    __device__ __forceinline__ int lane_here() const {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    }
    __device__ __forceinline__ void look_up() {
        const int64_t mine = next.first + threadIdx.x;
        row = (int)(mine < next.end ? mine : next.end - 1);
        if (g.scaled) row = g.scaled[row];
        if constexpr (GATHER) {
            const int l = lane_here();
#pragma unroll
            for (int c = 0; c < A::COPIES; ++c) {
                const unsigned r = (unsigned)next.first + A::row_of(c, wave, l), end = (unsigned)next.end;
                raw[c] = g.rows[r < end ? r : end - 1];
            }
        }
    }
    // a and b for the tile `next`, from its look-ups; rows outside are read
    // from row 0 and zeroed where they are stored
    __device__ __forceinline__ void point() {
        const int rows = (int)(next.end - next.first), n0 = next.col * TILE, l = lane_here();
        const int cols = g.N - n0 < TILE ? g.N - n0 : TILE;
        const int8_t *const W = g.W + next.e * g.sw + n0 * g.ldw;
        // leading dimensions in pairs
        a.init(uniform(reinterpret_cast<const char *>(g.X + (GATHER ? 0 : next.first * g.ldx))), g.ldx / 2, wave, l,
               [&](int c, int r) -> unsigned {
                   if constexpr (!GATHER) return r < rows ? r : rows - 1;
                   return raw[c] >= 0 && raw[c] < g.xrows ? raw[c] : 0;
               });
        b.init(uniform(reinterpret_cast<const char *>(W)), g.ldw / 2, wave, l,
               [&](int, int r) -> unsigned { return r < cols ? r : cols - 1; });
        kb = 0;
    }
    __device__ __forceinline__ bool start() {
        if (!product(next)) return false;
        look_up();
        point();
        return true;
    }
    // The scales go straight to LDS: waiting for them in registers would wait for the copies
    // in flight too (loads return in order).
    __device__ __forceinline__ void open() {
        turn ^= 1;
        if (!SUMS && wave * 64 < TILE) {
            Scales<TILE> &s = scales[turn];
            const int64_t n = (int64_t)now.col * TILE + threadIdx.x;
            const bool there = row >= 0 && row < g.xrows;
            s.there[threadIdx.x] = there;
            copy_lanes4(g.xs + (there ? row : 0), reinterpret_cast<char *>(s.x + wave * 64));
            copy_lanes4(g.ws + (int64_t)now.e * g.N + (n < g.N ? n : g.N - 1),
                        reinterpret_cast<char *>(s.w + wave * 64));
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
        // (the scales have landed: a barrier of the second or, of four stages, the third trip)
        // whether a row does not exist in X, or a column's scale could take its product with a
        // sum out of the range of normal numbers
        const Scales<TILE> &s = scales[turn];
        const int rows = (int)(now.end - now.first), cols = g.N - now.col * TILE;
        if (SUMS) {
            if (cols >= TILE) store_rows<PLAIN>(acc, s, rows, cols);
            else store_rows<CHECKED>(acc, s, rows, cols);
            return;
        }
        bool special = cols < TILE, extreme = false;
#pragma unroll
        for (int i = lane; i < RB * 32; i += 64) {
            special |= !s.there[(wave >> 1) * RB * 32 + i];
            extreme |= q8_extreme(s.w[(wave & 1) * RB * 32 + i]);
        }
        if (__any(extreme)) store_rows<EXTREME>(acc, s, rows, cols);
        else if (__any(special)) store_rows<CHECKED>(acc, s, rows, cols);
        else store_rows<PLAIN>(acc, s, rows, cols);
    }
    // PLAIN: every column and row of X exists; EXTREME: scales may be, else none is
    enum How { PLAIN, CHECKED, EXTREME };
    template <How HOW>
    __device__ __forceinline__ void store_rows(const i32x16 (&acc)[RB][RB], const Scales<TILE> &s, int rows,
                                               int cols) const {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        const int l = lane_here(), h = l >> 5, col0 = (wave & 1) * RB * 32;
        Out *const Y = static_cast<Out *>(g.Y) + now.first * g.ldy + now.col * TILE + col0;
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            const int row = ((wave >> 1) * RB + i) * 32 + (l & 31);
            if (row >= rows) continue;
            Out *const p = Y + row * g.ldy + (sizeof(T) == 4 ? 4 : 8) * h;
            const float x = SUMS ? 1.0f : s.x[row];
            const bool keep = HOW == PLAIN || SUMS || s.there[row];    // zeros for a row outside X, whatever W's scale
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                __builtin_amdgcn_sched_barrier(0);          // few values in flight: no registers to spare
#pragma unroll
                for (int r = 0; r < 16; r += 8) {
                    const int col = j * 32 + 2 * r;         // of 16 columns
                    const float *const ws = s.w + col0 + col + 4 * h;
                    const f32x4 w[2] = {*reinterpret_cast<const f32x4 *>(ws), *reinterpret_cast<const f32x4 *>(ws + 8)};
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int sum = acc[i][j][r + k];
                        const float m = w[k / 4][k % 4];
                        if constexpr (SUMS)
                            y[k] = __int_as_float(sum);
                        else if constexpr (HOW == EXTREME)
                            y[k] = q8_result(sum, m, x);
                        else
                            y[k] = (float)sum * m * x;          // the same
                    }
                    store8<HOW == PLAIN>(p + col, keep, cols - col0 - col, y);
                }
            }
        }
    }
    // y: columns 4 h .. 4 h + 3 and 8 + 4 h .. of 16, of which `cols` exist; p: the lane's first
    template <bool WHOLE>
    __device__ __forceinline__ void store8(Out *p, bool keep, int cols, float (&y)[8]) const {
        if constexpr (sizeof(T) == 4) {
            const int first = 4 * (lane >> 5);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = keep ? y[4 * q + k] : 0.0f;
                if (WHOLE || first + 8 * q + 4 <= cols) {
                    store_f32<4>(p + 8 * q, v);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (first + 8 * q + k < cols) p[8 * q + k] = v[k];
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
            if (!keep) w = u32x4{};
            const frag<T> f = __builtin_bit_cast(frag<T>, w);
            const int first = 8 * (lane >> 5);
            if (WHOLE || first + 8 <= cols) {
                *reinterpret_cast<vec<T, 8> *>(p) = f;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (first + k < cols) p[k] = f[k];
            }
        }
    }
};

// T int: the sums of a split.
template <typename T, int RB, int STAGES, bool GATHER>
__global__ __launch_bounds__(256, RB * STAGES == 4 ? 2 : 1) void q8_tiles_kernel(Q8Gemm g) {
    using Source = Q8Source<T, RB, STAGES, GATHER>;
    __shared__ __attribute__((aligned(1024))) char lds[STAGES * (Source::A::BYTES + Source::B::BYTES)];
    __shared__ TileList list;
    __shared__ __attribute__((aligned(16))) Scales<Source::TILE> scales[2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (Source::SUMS) to_split(g);
    list.fill(g, Source::TILE);
    Source src(g, list, scales, wave, lane);
    if (src.start()) run_tiles<i8pair, RB, STAGES, RB == 2 ? 2 : 1>(src, lds, wave);
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
hipError_t launch_q8_tiles(const Q8Gemm &g, Q8Tiles how, hipStream_t s) {
    auto run = [&](auto rb, auto stages) {
        constexpr int RB = decltype(rb)::value, STAGES = decltype(stages)::value, TILE = 64 * RB;
        const int64_t tiles = row_blocks_bound(g.R, g.E, TILE) * ((g.N + TILE - 1) / TILE);
        const unsigned grid = workgroups(tiles, RB * STAGES == 4 ? 2 : 1);
        if (g.rows) q8_tiles_kernel<T, RB, STAGES, true><<<grid, 256, 0, s>>>(g);
        else q8_tiles_kernel<T, RB, STAGES, false><<<grid, 256, 0, s>>>(g);
    };
    using std::integral_constant;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    if (how == Q8Tiles::LARGE) run(four, two);
    else if (how == Q8Tiles::SMALL) run(two, two);
    else run(two, four);
    return hipGetLastError();
}

}  // namespace
}  // namespace emu
