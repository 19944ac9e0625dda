// The grouped products of bfloat16 and half operands whose rows can be copied
// straight to LDS (16-byte alignment; see direct_gemm and direct_wgrad for the
// rule).
//
// A workgroup of 2 x 2 waves computes tiles of 64 RB x 64 RB (256 x 256 or
// 128 x 128), a wave RB x RB blocks of 32 x 32, by v_mfma 32 x 32 x 16.  A
// k-block of 64 indices of both operands is copied by global_load_lds into one
// of two LDS stages while the MFMAs of the other run; each lane names its own
// source, so the gather of token rows costs nothing and the 16-byte chunks are
// permuted on the way:
//   contiguous along the reduction (X; W stored N x K): 128 bytes a row, chunk q
//     of row r at q ^ (r / 2 % 8); read by ds_read_b128;
//   contiguous along the other direction (W stored K x N; both operands of the
//     matrix gradient): 128 RB bytes an index, chunk c of index k at c ^ 4 (k % 4);
//     read by ds_read_b64_tr_b16, which hands a lane four indices of one column.
// Either way the 16 lanes of a read phase (32 of the 8-byte read) touch every
// bank once.  k-blocks of 32 in four stages read 64-byte rows: 5 to 9 % slower.
//
// A wave's 256 accumulators leave one workgroup of 256 x 256 to a CU; its tiles run
// as one stream of k-blocks.  The copies of the next tile's first two k-blocks are in
// flight while a tile is stored, and the wait for the next ones is for the stores too.
// Measured in bfloat16: 131072 rows over 64 experts of 1024 x 2048, gathered, 557 to
// 610 us (0.9 to 1.0 PFLOP/s; a large library product reaches 1.47), of which the
// partly filled last tiles of the experts are 13 %; its matrix gradient over 65536
// rows 339 to 375 us (0.8 PFLOP/s).  The matrix instructions are busy for 49 and
// 33 % of the cycles, without an LDS bank conflict.  What a part costs, from copies of
// the kernels that leave it out (us, the product and the gradient):
//   as it is                  561   349
//   no stores                 520   299
//   no copies to LDS          423   278
//   no reads of fragments     501   349
//   matrix instructions only  346   213
// So the copies bound both, then the stores; the transposing reads cost nothing.
#pragma once

#include "gemm_common.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

template <typename T>
using frag = T __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4_ptr;

constexpr int BK = 64, SUBS = BK / 16;

__device__ __forceinline__ f32x16 mfma32(frag<bhalf> a, frag<bhalf> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(frag<half> a, frag<half> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Sixteen zero bytes that copies of rows outside read instead.
__device__ __attribute__((aligned(16))) float g_zero4[4];

// The copies and fragment reads of one operand of the tile: ROWS = 64 RB tile
// rows (or columns) by the indices of a k-block.
enum Mode { CONTIG, STRIDED };

template <int RB, int MODE>
struct Side;

template <int RB>
struct Side<RB, CONTIG> {
    static constexpr int ROWS = 64 * RB, BYTES = ROWS * BK * 2, COPIES = RB * BK / 32;        // per wave
    static constexpr int RS = BK * 2, Q = RS / 16;                              // a row's bytes, chunks
    static __device__ __forceinline__ int place(int r) { return r >> 1 & 7; }
    const char *base;               // uniform
    unsigned off[COPIES];
    int at[SUBS];                   // fragment offset per sub-step
    // tile row of a lane in copy c
    static __device__ __forceinline__ int row_of(int c, int wave, int lane) {
        return (wave * COPIES + c) * (1024 / RS) + lane / Q;
    }
    // row(c, r): the stored row of tile row r = row_of(c, ..)
    template <typename F>
    __device__ __forceinline__ void init(const char *base_, int64_t ld, int wave, int lane, F row) {
        base = base_;
#pragma unroll
        for (int c = 0; c < COPIES; ++c) {
            const int r = row_of(c, wave, lane);
            off[c] = (unsigned)((uint64_t)row(c, r) * (uint64_t)ld * 2) + ((lane % Q ^ place(r)) << 4);
        }
    }
    __device__ __forceinline__ void init_lane(int, int lane, int part) {
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
            at[s] = (part * 32 * RB + (lane & 31)) * RS + (((2 * s + (lane >> 5)) ^ place(lane & 31)) << 4);
    }
    __device__ __forceinline__ void copy(int c, int kb, char *stage, int wave) const {
        copy_lanes(base + (int64_t)kb * (BK * 2), off[c], stage + (wave * COPIES + c) * 1024);
    }
    template <typename T>
    __device__ __forceinline__ void read(frag<T> (&f)[RB], const char *stage, int s, int i) const {
        f[i] = *reinterpret_cast<const frag<T> *>(stage + at[s] + i * 32 * RS);
    }
};

// Transposing reads, and the chunk that a lane copies, of a [BK][ROWS] stage.
template <int RB>
struct StridedSide {
    static constexpr int ROWS = 64 * RB, RS = ROWS * 2, BYTES = BK * RS, COPIES = RB * BK / 32;
    static constexpr int LANES = RS / 16, PER = 64 / LANES;     // lanes per index, indices per copy
    int at[RB];
    __device__ __forceinline__ void init_reads(int lane, int part) {
        const int g = lane >> 4, i = lane & 15, k = 8 * (g >> 1) + (i >> 2);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int chunk = (part * RB + b) * 4 + 2 * (g & 1) + ((i & 3) >> 1);
            at[b] = k * RS + ((chunk ^ ((k & 3) * 4)) << 4) + (i & 1) * 8;
        }
    }
    // index within the k-block and byte within the row of copy c
    static __device__ __forceinline__ int index(int c, int wave, int lane) {
        return (wave * COPIES + c) * PER + lane / LANES;
    }
    static __device__ __forceinline__ int chunk(int c, int wave, int lane) {
        return (lane % LANES) ^ ((index(c, wave, lane) & 3) * 4);
    }
    template <typename T>
    __device__ __forceinline__ void read(frag<T> (&f)[RB], const char *stage, int s, int i) const {
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        char *const p = const_cast<char *>(stage) + at[i] + s * 16 * RS;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p + 4 * RS));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        f[i] = __builtin_bit_cast(frag<T>, v);
    }
};

template <int RB>
struct Side<RB, STRIDED> : StridedSide<RB> {
    using S = StridedSide<RB>;
    const char *base;
    int64_t step;                   // bytes from one k-block to the next
    unsigned off[S::COPIES];
    __device__ __forceinline__ void init_lane(int, int lane, int part) { S::init_reads(lane, part); }
    // cols: the columns that exist (rows have them up to a multiple of 8); copies past
    // them repeat the last ones
    __device__ __forceinline__ void init(const char *base_, int64_t ld, int64_t cols, int wave, int lane) {
        base = base_;
        step = ld * 2 * BK;
        const int last = (int)((cols + 7) / 8) - 1;
#pragma unroll
        for (int c = 0; c < S::COPIES; ++c) {
            const int q = S::chunk(c, wave, lane);
            off[c] = (unsigned)(S::index(c, wave, lane) * ld * 2) + ((q < last ? q : last) << 4);
        }
    }
    __device__ __forceinline__ void copy(int c, int kb, char *stage, int wave) const {
        copy_lanes(base + kb * step, off[c], stage + (wave * S::COPIES + c) * 1024);
    }
};

// Strided along a reduction over the `end` rows of an expert, through map where
// MAPPED: rows outside are zeros.
template <int RB, bool MAPPED>
struct RowSide : StridedSide<RB> {
    using S = StridedSide<RB>;
    static constexpr int WAVE_ROWS = S::COPIES * S::PER;        // rows of a k-block that a wave copies
    const char *base;
    unsigned ld2, col[2];           // a row's bytes; byte within a row for even and odd copies
    const __attribute__((address_space(4))) int *map;           // constant: read by scalar loads
    int64_t entries;
    int end, raw[WAVE_ROWS];        // row numbers of the k-block that is copied next
    const char *src[S::COPIES];     // sources of the k-block that is copied now
    int wave, lane;
    __device__ __forceinline__ void init_lane(int wave_, int lane_, int part) {
        wave = wave_;
        lane = lane_;
        S::init_reads(lane, part);
    }
    // base_: the tile's first column of row 0 of the operand (of the expert's first row without a map)
    __device__ __forceinline__ void init(const char *base_, int64_t ld, int64_t cols, const int *map_,
                                         int64_t entries_, int rows) {
        base = base_;
        ld2 = (unsigned)(ld * 2);
        map = (const __attribute__((address_space(4))) int *)map_;
        entries = entries_;
        end = rows;
        const int last = (int)((cols + 7) / 8) - 1;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int q = S::chunk(c, wave, lane);
            col[c] = (unsigned)(q < last ? q : last) << 4;
        }
    }
    // reads the row numbers of k-block kb
    __device__ __forceinline__ void preload(int kb) {
        if constexpr (MAPPED) {
            const int k = kb * BK + wave * WAVE_ROWS;
            if (k + WAVE_ROWS <= end) {
#pragma unroll
                for (int i = 0; i < WAVE_ROWS; ++i) raw[i] = map[k + i];
            } else {
#pragma unroll
                for (int i = 0; i < WAVE_ROWS; ++i) raw[i] = k + i < end ? map[k + i] : -1;
            }
        }
    }
    // the sources of k-block kb, whose row numbers have been read
    __device__ __forceinline__ void resolve(int kb) {
#pragma unroll
        for (int c = 0; c < S::COPIES; ++c) {
            int r;
            bool there;
            if constexpr (MAPPED) {
                r = raw[c * S::PER];
#pragma unroll
                for (int i = 1; i < S::PER; ++i) r = lane >= i * S::LANES ? raw[c * S::PER + i] : r;
                there = r >= 0 && r < entries;
            } else {
                r = kb * BK + S::index(c, wave, lane);
                there = r < end;
            }
            const char *const p = base + (uint64_t)(unsigned)r * ld2 + col[c & 1];
            src[c] = there ? p : reinterpret_cast<const char *>(g_zero4);
        }
    }
    __device__ __forceinline__ void copy(int c, int, char *stage, int) const {
        copy_lanes(src[c], stage + (wave * S::COPIES + c) * 1024);
    }
};

// Runs a workgroup's tiles.  Their k-blocks form one stream through two LDS
// stages: entering a trip the first fragments of its k-block are in registers
// and the copies of the next k-block are in flight.  Sub-steps 0 to 2 run on the
// trip's stage; then every wave has read all of it and the next k-block has
// landed, and during sub-step 3 the copies of the k-block after that start and
// the first fragments of the next one are read.  At the end of a tile those are
// the next tile's, so that its results are stored while the copies run.
//   src.a, src.b     the operands of the tile whose k-blocks are copied next
//   src.open()       a tile starts (its k-blocks 0 and 1 are copied)
//   src.trip()       a trip starts
//   src.landed()     no copy is in flight; the next one follows
//   src.copied()     the copies of a k-block have been started
//   src.blocks()     k-blocks of the current tile, at least 2
//   src.close(acc)   the tile is done; false: it was the last
template <typename T, int RB, typename Source>
__device__ __forceinline__ void run_tiles(Source &src, char *lds, int wave) {
    using A = decltype(src.a);
    using B = decltype(src.b);
    constexpr int STAGE = A::BYTES + B::BYTES, COPIES = A::COPIES + B::COPIES, BLOCKS = RB * RB;
    f32x16 acc[RB][RB];
    auto copy = [&](int c, char *stage) {
        if (c < A::COPIES) src.a.copy(c, src.kb, stage, wave);
        else src.b.copy(c - A::COPIES, src.kb, stage + A::BYTES, wave);
    };
    struct Frags {
        frag<T> a[RB], b[RB];
    } f[2];
    auto read = [&](Frags &g, const char *stage, int s, int u) {
        if (u < RB) src.b.template read<T>(g.b, stage + A::BYTES, s, u);
        else src.a.template read<T>(g.a, stage, s, u - RB);
    };
    for (int i = 0; i < 2; ++i) {
        src.trip();
        src.landed();
        static_for<COPIES>([&](auto c) { copy(c, lds + i * STAGE); });
        src.copied();
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
    __syncthreads();
    static_for<2 * RB>([&](auto u) { read(f[0], lds, 0, u); });
    int at = 0;                     // the stage of the trip's k-block
    do {
        src.open();
        const int KB = src.blocks();
        auto trip = [&](auto first) {
            char *const cur = lds + uniform(at), *const nxt = lds + uniform(STAGE - at);
            // MFMA t, then the reads of the next sub-step whose turn it is, then copies
            auto step = [&](auto s_c, const char *from, auto copies) {
                constexpr int s = decltype(s_c)::value;
                Frags &g = f[s & 1], &n = f[1 - (s & 1)];
                static_for<BLOCKS>([&](auto t_c) {
                    constexpr int t = decltype(t_c)::value;
                    f32x16 &c = acc[t / RB][t % RB];
                    c = mfma32(g.b[t % RB], g.a[t / RB], decltype(first)::value && s == 0 ? f32x16{} : c);
                    order_fence();
                    static_for<2 * RB>([&](auto u) {
                        if constexpr (u * BLOCKS / (2 * RB) == t) read(n, from, (s + 1) % SUBS, u);
                    });
                    order_fence();
                    if constexpr (decltype(copies)::value)
                        static_for<COPIES>([&](auto i) {
                            if constexpr (i * BLOCKS / COPIES == t) copy(i, cur);
                        });
                    order_fence();
                });
            };
            src.trip();
            static_for<SUBS - 1>([&](auto i) { step(i, cur, std::false_type{}); });
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            pipeline_barrier();
            src.landed();
            step(std::integral_constant<int, SUBS - 1>{}, nxt, std::true_type{});
            __builtin_amdgcn_sched_barrier(0);
            src.copied();
            at = STAGE - at;
        };
        trip(std::true_type{});
        for (int kb = 1; kb < KB; ++kb) trip(std::false_type{});
    } while (src.close(acc));
    // the last copies are not read: they must land before the workgroup ends
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// acc to C; keep(i): the lane's row of row block i has its sum (else zero).  The columns are
// the MFMA's rows: register r of lane l is column 8 (r / 4) + 4 (l / 32) + r % 4
// of row l % 32 of its block.  An exchange between the lane halves gives each
// eight neighbouring columns of its row, one 16-byte store.
template <typename T, int RB, typename F>
__device__ __forceinline__ void store(const f32x16 (&acc)[RB][RB], int wave, int lane, int rows,
                                      int cols, T *__restrict__ C, int64_t ldc, F keep) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    auto pack = [](float x, float y) {
        const t2 v = {(T)x, (T)y};
        return __builtin_bit_cast(unsigned, v);
    };
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int row = ((wave >> 1) * RB + i) * 32 + (lane & 31);
        const bool there = row < rows, k = there && keep(i);
        T *const p = C + row * ldc;
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                __builtin_amdgcn_sched_barrier(0);      // few values in flight: no registers to spare
                const f32x16 &v = acc[i][j];
                const u32x2 x = __builtin_amdgcn_permlane32_swap(pack(v[r], v[r + 1]), pack(v[r + 4], v[r + 5]),
                                                                 false, false);
                const u32x2 y = __builtin_amdgcn_permlane32_swap(pack(v[r + 2], v[r + 3]),
                                                                 pack(v[r + 6], v[r + 7]), false, false);
                u32x4 w = {x[0], y[0], x[1], y[1]};
                if (!k) w = u32x4{};
                const int col = ((wave & 1) * RB + j) * 32 + 2 * r + 8 * (lane >> 5);
                if (!there) continue;
                if (col + 8 <= cols) {
                    *reinterpret_cast<vec<T, 8> *>(p + col) = __builtin_bit_cast(frag<T>, w);
                } else {
                    const frag<T> e = __builtin_bit_cast(frag<T>, w);
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (col + c < cols) p[col + c] = e[c];
                }
            }
    }
}

// acc to FP32 C, whose rows have their columns up to a multiple of four.
template <int RB>
__device__ __forceinline__ void store_sums(const f32x16 (&acc)[RB][RB], int wave, int lane, int rows, int cols,
                                           float *__restrict__ C, int64_t ldc) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int row = ((wave >> 1) * RB + i) * 32 + (lane & 31);
        if (row >= rows) continue;
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int col = ((wave & 1) * RB + j) * 32 + 2 * r + 4 * (lane >> 5);
                const f32x16 &v = acc[i][j];
                const f32x4 w = {v[r], v[r + 1], v[r + 2], v[r + 3]};
                if (col < cols) *reinterpret_cast<f32x4 *>(C + row * ldc + col) = w;
            }
    }
}

constexpr int LIST = 64;            // most tiles of a workgroup

// The row tiles w, w + workgroups, ... of a grouped product, found before the
// first of them runs and kept in LDS (searching between tiles would leave the
// matrix cores idle, and its control flow costs the accumulators registers).
struct TileList {
    int4 tile[LIST + 1];            // expert, first row, end, column tile; ends with expert -1
    __device__ __forceinline__ void fill(const GroupedGemm &g, int rows) {
        if (threadIdx.x < 64) {
            const RowTiles tiles(g.offsets, g.E, g.R, rows, (g.N + rows - 1) / rows);
            for (int i = 0; i <= LIST; ++i) {
                RowTile t = i < LIST ? tiles.of_workgroup(blockIdx.x + (int64_t)i * gridDim.x) : RowTile{-1, 0, 0, 0};
                if (threadIdx.x == 0) tile[i] = {t.e, (int)t.first, (int)t.end, t.col};
                if (t.e < 0) break;
            }
        }
        __syncthreads();
    }
    __device__ __forceinline__ RowTile at(int i) const {
        const int4 t = tile[i];
        return {uniform(t.x), uniform(t.y), uniform(t.z), uniform(t.w)};
    }
};

template <typename T, int RB, bool TB, bool GATHER>
struct GemmSource {
    static constexpr int TILE = 64 * RB;
    using A = Side<RB, CONTIG>;
    using B = Side<RB, TB ? CONTIG : STRIDED>;
    const GroupedGemm &g;
    const TileList &list;
    int i;                          // list entry of `next`
    RowTile now, next;              // the tile that is computed, and the one after
    A a;
    B b;
    int kb, KB, wave, lane;
    int raw[A::COPIES], kept[RB];   // look-ups: of the next tile's copies; of the rows to store

    __device__ __forceinline__ GemmSource(const GroupedGemm &g_, const TileList &list_, int wave_, int lane_)
        : g(g_), list(list_), i(0), wave(wave_), lane(lane_) {
        a.init_lane(wave, lane, wave >> 1);
        b.init_lane(wave, lane, wave & 1);
        KB = g.K / BK;
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
        const T *const X = static_cast<const T *>(g.X), *const W = static_cast<const T *>(g.W) + next.e * g.sw;
        a.init(reinterpret_cast<const char *>(X + (GATHER ? 0 : next.first * g.ldx)), g.ldx, wave, lane,
               [&](int c, int r) -> unsigned {
                   if constexpr (!GATHER) return r < rows ? r : rows - 1;
                   return raw[c] >= 0 && raw[c] < g.xrows ? raw[c] : 0;
               });
        if constexpr (TB)
            b.init(reinterpret_cast<const char *>(W + n0 * g.ldw), g.ldw, wave, lane,
                   [&](int, int r) -> unsigned { return r < cols ? r : cols - 1; });
        else
            b.init(reinterpret_cast<const char *>(W + n0), g.ldw, cols, wave, lane);
        kb = 0;
    }
    __device__ __forceinline__ bool start() {
        if (!product(next)) return false;
        look_up();
        point();
        return true;
    }
    __device__ __forceinline__ void open() {
        if constexpr (GATHER) {
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const int r = (int)now.first + ((wave >> 1) * RB + j) * 32 + (lane & 31);
                kept[j] = g.rows[r < now.end ? r : (int)now.end - 1];
            }
        }
        // after the last product its own k-blocks are copied again, unused
        const RowTile t = list.at(i + 1);
        if (product(t)) next = t;
        ++i;
        look_up();
    }
    __device__ __forceinline__ void trip() {}
    __device__ __forceinline__ void landed() {
        if (kb == KB) point();
    }
    __device__ __forceinline__ void copied() { ++kb; }
    __device__ __forceinline__ int blocks() const { return KB; }
    __device__ __forceinline__ bool close(const f32x16 (&acc)[RB][RB]) {
        const int n0 = now.col * TILE, cols = g.N - n0 < TILE ? g.N - n0 : TILE;
        store<T, RB>(acc, wave, lane, (int)(now.end - now.first), cols,
                     static_cast<T *>(g.Y) + now.first * g.ldy + n0, g.ldy,
                     [&](int j) { return !GATHER || (kept[j] >= 0 && kept[j] < g.xrows); });
        now = next;
        return product(list.at(i));
    }
};

template <typename T, int RB, bool TB, bool GATHER>
__global__ __launch_bounds__(256, RB == 4 ? 1 : 2) void gemm16_kernel(GroupedGemm g) {
    using Source = GemmSource<T, RB, TB, GATHER>;
    __shared__ __attribute__((aligned(1024))) char lds[2 * (Source::A::BYTES + Source::B::BYTES)];
    __shared__ TileList list;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    list.fill(g, Source::TILE);
    Source src(g, list, wave, lane);
    if (src.start()) run_tiles<T, RB>(src, lds, wave);
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

// The tiles w, w + workgroups, ... of the matrices' gradients.
template <typename T, int RB, int MAPPED>        // the operand that goes through a map: 0 none, 1 P, 2 Q
struct WgradSource {
    static constexpr int TILE = 64 * RB;
    static constexpr bool PIECES = RB == 2;     // an expert's rows may be in pieces (the others have no registers to spare)
    using A = RowSide<RB, MAPPED == 1>;
    using B = RowSide<RB, MAPPED == 2>;
    const GroupedWgrad &g;
    const int mt, nt;
    int id, end;                    // the next tile, and the end of the XCD's
    struct Tile {
        int e, m, n, lo, rows;      // e: piece of an expert, -1 for no tile
    } now, next;
    A a;
    B b;
    int kb, KB;                     // of the tile that a and b stand for

    __device__ __forceinline__ WgradSource(const GroupedWgrad &g_, int wave, int lane)
        : g(g_), mt((g_.M + TILE - 1) / TILE), nt((g_.N + TILE - 1) / TILE) {
        // an XCD has a contiguous run of tiles, so of experts, and its workgroups take them in
        // turn.  The runs take the same time (unevenly loaded experts: 401 -> 388 us); where
        // a workgroup has one tile at most, they are of equal length.
        const int64_t each = (int64_t)(PIECES ? g.pieces : 1) * mt * nt, total = g.E * each, per = (total + 7) / 8;
        const int x = blockIdx.x % 8;
        const bool even = total <= gridDim.x;
        const int64_t first = even ? x * per : first_tile_of_xcd(g.offsets, g.E, g.R, each, x);
        end = uniform(even ? (first + per < total ? first + per : total)
                           : first_tile_of_xcd(g.offsets, g.E, g.R, each, x + 1));
        id = uniform(first) + blockIdx.x / 8;
        a.init_lane(wave, lane, wave >> 1);
        b.init_lane(wave, lane, wave & 1);
        now = next = tile();
    }
    __device__ __forceinline__ Tile tile() const {
        if (id >= end) return {-1, 0, 0, 0, 0};
        const int e = id / (mt * nt), r = id % (mt * nt);
        int64_t lo, hi;
        expert_rows(g.offsets, g.E, g.R, PIECES ? e / g.pieces : e, lo, hi);
        if constexpr (PIECES) piece_rows(e % g.pieces, g.pieces, lo, hi);
        return {uniform(e), uniform(r % mt * TILE), uniform(r / mt * TILE), uniform(lo), uniform(hi - lo)};
    }
    // at least two, the missing ones zeros
    static __device__ __forceinline__ int blocks_of(const Tile &t) {
        const int n = (t.rows + BK - 1) / BK;
        return n < 2 ? 2 : n;
    }
    __device__ __forceinline__ void point() {
        const Tile &t = next;
        const int m = g.M - t.m < TILE ? g.M - t.m : TILE, n = g.N - t.n < TILE ? g.N - t.n : TILE;
        a.init(reinterpret_cast<const char *>(static_cast<const T *>(g.P) + t.m + (MAPPED == 1 ? 0 : t.lo * g.ldp)),
               g.ldp, m, MAPPED == 1 ? g.prow + t.lo : nullptr, g.prows, t.rows);
        b.init(reinterpret_cast<const char *>(static_cast<const T *>(g.Q) + t.n + (MAPPED == 2 ? 0 : t.lo * g.ldq)),
               g.ldq, n, MAPPED == 2 ? g.qrow + t.lo : nullptr, g.qrows, t.rows);
        kb = 0;
        KB = blocks_of(t);
        a.preload(0);
        b.preload(0);
    }
    __device__ __forceinline__ bool start() {
        if (next.e < 0) return false;
        point();
        return true;
    }
    __device__ __forceinline__ void open() {
        id += gridDim.x / 8;
        next = tile();
    }
    __device__ __forceinline__ void trip() {
        if (kb == KB) {
            if (next.e >= 0) point();
            else kb = KB - 1;       // nothing follows: the last k-block again
        }
        a.resolve(kb);
        b.resolve(kb);
        if (kb + 1 < KB) {
            a.preload(kb + 1);
            b.preload(kb + 1);
        }
    }
    __device__ __forceinline__ void landed() {}
    __device__ __forceinline__ void copied() { ++kb; }
    __device__ __forceinline__ int blocks() const { return blocks_of(now); }
    __device__ __forceinline__ bool close(const f32x16 (&acc)[RB][RB]) {
        const int m = g.M - now.m < TILE ? g.M - now.m : TILE, n = g.N - now.n < TILE ? g.N - now.n : TILE;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t at = now.e * g.sw + now.m * g.ldw + now.n;
        if (PIECES && g.pieces > 1) store_sums<RB>(acc, wave, lane, m, n, static_cast<float *>(g.dW) + at, g.ldw);
        else store<T, RB>(acc, wave, lane, m, n, static_cast<T *>(g.dW) + at, g.ldw, [](int) { return true; });
        now = next;
        return now.e >= 0;
    }
};

template <typename T, int RB, int MAPPED>
__global__ __launch_bounds__(256, RB == 4 ? 1 : 2) void wgrad16_kernel(GroupedWgrad g) {
    using Source = WgradSource<T, RB, MAPPED>;
    __shared__ __attribute__((aligned(1024))) char lds[2 * (Source::A::BYTES + Source::B::BYTES)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Source src(g, wave, lane);
    if (src.start()) run_tiles<T, RB>(src, lds, wave);
}

// Workgroups of a launch over `tiles` tiles: as many as run at a time (more
// where that would be over half of LIST tiles each), a multiple of 8 (an XCD's tiles
// stay its own).
unsigned workgroups(int64_t tiles, int per_cu) {
    int64_t most = persistent_workgroups(device_cu_count()) * (int64_t)per_cu;
    if (most * (LIST / 2) < tiles) most = tiles / (LIST / 2) + 1;
    return (unsigned)(((tiles < most ? tiles : most) + 7) / 8 * 8);
}

template <typename T>
hipError_t launch_gemm16(const GroupedGemm &g, int tile, hipStream_t s) {
    auto run = [&](auto rb) {
        constexpr int RB = decltype(rb)::value, TILE = 64 * RB;
        const int64_t tiles = row_blocks_bound(g.R, g.E, TILE) * ((g.N + TILE - 1) / TILE);
        const unsigned grid = workgroups(tiles, RB == 4 ? 1 : 2);
        auto layout = [&](auto tb) {
            if (g.rows) gemm16_kernel<T, RB, decltype(tb)::value, true><<<grid, 256, 0, s>>>(g);
            else gemm16_kernel<T, RB, decltype(tb)::value, false><<<grid, 256, 0, s>>>(g);
        };
        if (g.transb) layout(std::true_type{});
        else layout(std::false_type{});
    };
    if (tile == 256) run(std::integral_constant<int, 4>{});
    else run(std::integral_constant<int, 2>{});
    return hipGetLastError();
}

template <typename T>
hipError_t launch_wgrad16(const GroupedWgrad &g, int tile, hipStream_t s) {
    auto run = [&](auto rb) {
        constexpr int RB = decltype(rb)::value, TILE = 64 * RB;
        const int64_t tiles = (int64_t)g.E * g.pieces * ((g.M + TILE - 1) / TILE) * ((g.N + TILE - 1) / TILE);
        const unsigned grid = workgroups(tiles, RB == 4 ? 1 : 2);
        if constexpr (RB == 4) {
            if (g.prow) return wgrad16_kernel<T, RB, 1><<<grid, 256, 0, s>>>(g);
            if (g.qrow) return wgrad16_kernel<T, RB, 2><<<grid, 256, 0, s>>>(g);
        }
        wgrad16_kernel<T, RB, 0><<<grid, 256, 0, s>>>(g);
    };
    if (tile == 256) run(std::integral_constant<int, 4>{});
    else run(std::integral_constant<int, 2>{});
    return hipGetLastError();
}

}  // namespace
}  // namespace emu
