// The grouped products of FP32 operands on full tiles: six BF16 component
// products (Eq. fp32six), split where they are staged.
//
// A workgroup of eight waves computes a tile of 256 x 128 (or of 192 or 128 rows), a
// k-block of 32 indices at a time.  The FP32 entries of the k-block after the next
// are loaded into registers (24 of a lane), split into three BF16 components
// (v_cvt_pk_bf16_f32, an exact subtraction; five instructions an entry) and
// written to the LDS stage that the k-block before has released: every entry is
// split once for the whole tile, nothing goes through memory, and gathered
// rows, strides and odd extents cost nothing extra.  Two waves share a SIMD
// (waves w and w + 4): the one splits and writes while the other's matrix
// instructions run, then they change over; a k-block is one barrier.  A0B0 goes
// to one accumulator set, the five smaller products to another, added at the
// end (see grouped.hip).
//
// Bytes in LDS per k-block at 256 x 128: 74 KB written, 196 KB read in the 3072
// cycles of its MFMAs, so the matrix instructions bound it.
#include "gemm_common.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));
constexpr int BN = 128, BK = 32, THREADS = 512, PL = 3;

// What loads of entries outside read: a row of zeros as wide as a tile.
__device__ __attribute__((aligned(16))) float g_zeros[256];

// Where chunk q (eight indices) of tile row r lies in a plane of a stage.
__device__ __forceinline__ int chunk_at(int r, int q) { return r * 64 + ((q ^ swz(r)) << 4); }

__device__ __forceinline__ void split_to(char *dst, int plane, f32x8 x) {
#pragma unroll
    for (int c = 0; c < PL; ++c) {
        const bf16x8 h = __builtin_convertvector(x, bf16x8);
        *reinterpret_cast<bf16x8 *>(dst + c * plane) = h;
        if (c + 1 < PL) x = x - __builtin_convertvector(h, f32x8);
    }
}

// Whether this wave has its unit i of ROWS tile rows (192 rows are 12 units of
// a wave, the last four of waves 0 to 3).
template <int ROWS>
__device__ __forceinline__ bool has_unit(int i) {
    return ROWS / 16 % 8 == 0 || i < ROWS / 128 || __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < 4;
}

// The loads of one operand, ROWS tile rows by the k-block, UNITS runs of eight
// indices to a thread.  Contiguous along the reduction: row(r) gives the stored
// row of tile row r or -1 (zeros).
template <int ROWS>
struct ContigLoads {
    static constexpr int UNITS = (ROWS * 4 + THREADS - 1) / THREADS;
    f32x8 x[UNITS];
    const float *src[UNITS];
    bool there[UNITS];
    template <typename F>
    __device__ __forceinline__ void init(const float *base, int64_t ld, F row) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = threadIdx.x + THREADS * i;
            const int64_t r = has_unit<ROWS>(i) ? row(u >> 2) : -1;
            there[i] = r >= 0;
            src[i] = base + (there[i] ? r * ld : 0) + (u & 3) * 8;
        }
    }
    __device__ __forceinline__ void load(int k0, int K) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            if (!has_unit<ROWS>(i)) continue;
            const float *const p = src[i] + k0;
            if (k0 + BK <= K) {
                x[i] = *reinterpret_cast<const vec<float, 8> *>(p);
            } else {
                const int left = K - k0 - ((threadIdx.x + THREADS * i) & 3) * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = j < left ? p[j] : 0.0f;
            }
        }
    }
    __device__ __forceinline__ void write(char *stage) const {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = threadIdx.x + THREADS * i;
            if (has_unit<ROWS>(i)) split_to(stage + chunk_at(u >> 2, u & 3), ROWS * 64, there[i] ? x[i] : f32x8{});
        }
    }
};

// Contiguous along the tile rows (columns of W stored K x N; the operands of
// the matrix gradient): a wave takes 64 tile rows of eight indices, whose stored
// rows are uniform over the wave; look-ups in `map` are scalar loads.
template <int ROWS, bool MAP>
struct StridedLoads {
    static constexpr int GROUPS = ROWS / 64, UNITS = (GROUPS * 4 + 7) / 8;
    f32x8 x[UNITS];
    const float *base;
    unsigned ld, entries;
    const __attribute__((address_space(4))) int *map;
    unsigned col[UNITS];            // byte of the lane's column
    int q[UNITS], r[UNITS];
    __device__ __forceinline__ void init(const float *base_, int64_t ld_, const int *map_, int64_t entries_,
                                         int rows) {
        base = base_;
        ld = (unsigned)ld_;
        map = (const __attribute__((address_space(4))) int *)map_;
        entries = MAP ? (unsigned)entries_ : 0xFFFFFFFFu;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = wave + 8 * i;
            q[i] = u / GROUPS;
            r[i] = u % GROUPS * 64 + lane;
            col[i] = (r[i] < rows ? r[i] : rows - 1) * 4;
        }
    }
    // the lane's entry of a row: 64-bit base in scalar registers, 32-bit offset
    __device__ __forceinline__ float at_row(const float *row, int i) const {
        asm volatile("" : "+s"(row));
        return *reinterpret_cast<const float *>(reinterpret_cast<const char *>(row) + col[i]);
    }
    __device__ __forceinline__ void load(int k0, int K) {
        if (MAP || k0 + BK > K) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                if (!has_unit<ROWS>(i)) continue;
                const int k = k0 + q[i] * 8;
                int at[8];
                if (MAP && k0 + BK <= K) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) at[j] = map[k + j];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) at[j] = k + j < K ? (MAP ? map[k + j] : k + j) : -1;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool there = (unsigned)at[j] < entries;
                    x[i][j] = at_row(there ? base + (uint64_t)(unsigned)at[j] * ld : g_zeros, i);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                if (!has_unit<ROWS>(i)) continue;
                const float *row = base + (uint64_t)(unsigned)(k0 + q[i] * 8) * ld;
#pragma unroll
                for (int j = 0; j < 8; ++j, row += ld) x[i][j] = at_row(row, i);
            }
        }
    }
    __device__ __forceinline__ void write(char *stage) const {
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
            if (has_unit<ROWS>(i)) split_to(stage + chunk_at(r[i], q[i]), ROWS * 64, x[i]);
    }
};

// C = A B^T of the tile, rows x cols of it stored.  WM x WN waves of RB x CB
// blocks of 32 x 32.
template <int WM, int WN, int RB, int CB, typename A, typename B>
__device__ __forceinline__ void tile_product(A &a, B &b, int K, int rows, int cols, float *__restrict__ C,
                                             int64_t ldc, char *lds) {
    constexpr int AROWS = 32 * WM * RB, STAGE = PL * (AROWS + BN) * 64;
    static_assert(WM * WN == 8 && WN * CB * 32 == BN, "eight waves, 128 columns");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const bool early = wave < 4;
    f32x16 hi[RB][CB], lo[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) hi[i][j] = lo[i][j] = f32x16{};
    if (K > 0) {
        a.load(0, K);
        b.load(0, K);
        a.write(lds);
        b.write(lds + PL * AROWS * 64);
        if (BK < K) {
            a.load(BK, K);
            b.load(BK, K);
        }
    }
    const int fa = wm * RB * 32 * 64, fb = PL * AROWS * 64 + wn * CB * 32 * 64;
    int at = 0;
    for (int k0 = 0; k0 < K; k0 += BK) {
        __syncthreads();
        char *const cur = lds + at, *const nxt = lds + (STAGE - at);
        auto produce = [&]() __attribute__((always_inline)) {
            if (k0 + BK < K) {
                a.write(nxt);
                b.write(nxt + PL * AROWS * 64);
            }
            if (k0 + 2 * BK < K) {
                a.load(k0 + 2 * BK, K);
                b.load(k0 + 2 * BK, K);
            }
        };
        if (early) produce();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int off = frag_offset(lane, s);
            bf16x8 x[PL][RB], y[PL][CB];
#pragma unroll
            for (int c = 0; c < PL; ++c) {
#pragma unroll
                for (int i = 0; i < RB; ++i) x[c][i] = lds_frag(cur + fa + (c * AROWS + i * 32) * 64, off);
#pragma unroll
                for (int j = 0; j < CB; ++j) y[c][j] = lds_frag(cur + fb + (c * BN + j * 32) * 64, off);
            }
            // the sum of the planes' numbers descending, so that hi comes last: product-major
#pragma unroll
            for (int c = 0; c < PL; ++c)
#pragma unroll
                for (int d = 0; c + d < PL; ++d)
#pragma unroll
                    for (int i = 0; i < RB; ++i)
#pragma unroll
                        for (int j = 0; j < CB; ++j) {
                            f32x16 &acc = c + d == 0 ? hi[i][j] : lo[i][j];
                            acc = mfma(x[c][i], y[d][j], acc);
                        }
        }
        if (!early) produce();
        at = STAGE - at;
    }
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            const int col = (wn * CB + j) * 32 + (lane & 31);
            if (col >= cols) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = (wm * RB + i) * 32 + acc_row(r) + acc_lrow(lane);
                if (row < rows) C[row * ldc + col] = hi[i][j][r] + lo[i][j][r];
            }
        }
}

template <int AROWS>
constexpr int lds_bytes() { return 2 * PL * (AROWS + BN) * 64; }

template <int WM, int WN, int RB, int CB, bool TB>
__global__ __launch_bounds__(THREADS, 2) void gemm32_kernel(GroupedGemm g) {
    constexpr int AROWS = 32 * WM * RB;
    __shared__ __attribute__((aligned(1024))) char lds[lds_bytes<AROWS>()];
    const RowTile t = RowTiles(g.offsets, g.E, g.R, AROWS, (g.N + BN - 1) / BN).of_workgroup(blockIdx.x);
    if (t.e < 0) return;
    const int rows = (int)(t.end - t.first), n0 = t.col * BN, cols = g.N - n0 < BN ? g.N - n0 : BN;
    const bool none = t.e == g.E;               // rows of no expert: an empty reduction gives their zeros
    const float *const X = static_cast<const float *>(g.X);
    const float *const W = static_cast<const float *>(g.W) + (none ? 0 : t.e * g.sw);
    ContigLoads<AROWS> a;
    a.init(X, g.ldx, [&](int r) -> int64_t {
        const int64_t i = t.first + (r < rows ? r : rows - 1);
        if (!g.rows) return i;
        const int64_t m = g.rows[i];
        return m < g.xrows ? m : -1;
    });
    float *const C = static_cast<float *>(g.Y) + t.first * g.ldy + n0;
    const int K = none ? 0 : g.K;
    if constexpr (TB) {
        ContigLoads<BN> b;
        b.init(W + n0 * g.ldw, g.ldw, [&](int r) -> int64_t { return r < cols ? r : cols - 1; });
        tile_product<WM, WN, RB, CB>(a, b, K, rows, cols, C, g.ldy, lds);
    } else {
        StridedLoads<BN, false> b;
        b.init(W + n0, g.ldw, nullptr, 0, cols);
        tile_product<WM, WN, RB, CB>(a, b, K, rows, cols, C, g.ldy, lds);
    }
}

template <int WM, int WN, int RB, int CB, int MAPPED>  // the operand that goes through a map: 0 none, 1 P, 2 Q
__global__ __launch_bounds__(THREADS, 2) void wgrad32_kernel(GroupedWgrad g) {
    constexpr int AROWS = 32 * WM * RB;
    __shared__ __attribute__((aligned(1024))) char lds[lds_bytes<AROWS>()];
    const int mt = (g.M + AROWS - 1) / AROWS, nt = (g.N + BN - 1) / BN;
    // an XCD takes a contiguous run of tiles, so of experts
    const int64_t total = (int64_t)g.E * mt * nt, per = (total + 7) / 8;
    const int64_t id = blockIdx.x % 8 * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return;
    const int e = uniform(id / (mt * nt)), r = uniform(id % (mt * nt));
    const int m0 = r % mt * AROWS, n0 = r / mt * BN;
    const int rows = g.M - m0 < AROWS ? g.M - m0 : AROWS, cols = g.N - n0 < BN ? g.N - n0 : BN;
    int64_t lo, hi;
    expert_rows(g.offsets, g.E, g.R, e, lo, hi);
    lo = uniform(lo);
    const int K = uniform(hi - lo);
    StridedLoads<AROWS, MAPPED == 1> a;
    StridedLoads<BN, MAPPED == 2> b;
    a.init(static_cast<const float *>(g.P) + m0 + (MAPPED == 1 ? 0 : lo * g.ldp), g.ldp,
           MAPPED == 1 ? g.prow + lo : nullptr, g.prows, rows);
    b.init(static_cast<const float *>(g.Q) + n0 + (MAPPED == 2 ? 0 : lo * g.ldq), g.ldq,
           MAPPED == 2 ? g.qrow + lo : nullptr, g.qrows, cols);
    tile_product<WM, WN, RB, CB>(a, b, K, rows, cols, static_cast<float *>(g.dW) + e * g.sw + m0 * g.ldw + n0,
                                 g.ldw, lds);
}

}  // namespace

namespace {

// f(waves and blocks) of the tile height whose launch takes least time: rounds
// of one workgroup per CU, each as long as its tile's products take.  At 8192 x
// 8192 x 8192 tiles of 256, 192 and 128 rows measured 206, 188 and 174 TFLOP/s,
// so a round of them takes 100, 83 and 59 units; which height wins is a matter
// of how the last round is filled.  blocks(h): row blocks of that height.
template <typename F, typename G>
void with_height(int64_t col_tiles, F blocks, G &&f) {
    using std::integral_constant;
    const int cus = device_cu_count();
    auto time = [&](int h, int units) { return (blocks(h) * col_tiles + cus - 1) / cus * units; };
    const int64_t t256 = time(256, 100), t192 = time(192, 83), t128 = time(128, 59);
    const int best = t256 <= t192 && t256 <= t128 ? 256 : (t192 <= t128 ? 192 : 128);
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 3> three;
    const integral_constant<int, 4> four;
    if (best == 256) f(four, two, two, two);
    else if (best == 192) f(two, four, three, one);
    else f(four, two, one, two);
}

}  // namespace

hipError_t launch_gemm32(const GroupedGemm &g, hipStream_t s) {
    const int64_t nt = (g.N + BN - 1) / BN;
    // an expert's last block is half full on average
    with_height(nt, [&](int h) { return (g.R + (int64_t)g.E * h / 2) / h; }, [&](auto wm, auto wn, auto rb, auto cb) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, RB = decltype(rb)::value, CB = decltype(cb)::value;
        const unsigned grid = (unsigned)((row_blocks_bound(g.R, g.E, 32 * WM * RB) * nt + 7) / 8 * 8);
        if (g.transb) gemm32_kernel<WM, WN, RB, CB, true><<<grid, THREADS, 0, s>>>(g);
        else gemm32_kernel<WM, WN, RB, CB, false><<<grid, THREADS, 0, s>>>(g);
    });
    return hipGetLastError();
}

hipError_t launch_wgrad32(const GroupedWgrad &g, hipStream_t s) {
    const int64_t nt = (g.N + BN - 1) / BN;
    with_height(nt * g.E, [&](int h) { return (g.M + h - 1) / h; }, [&](auto wm, auto wn, auto rb, auto cb) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, RB = decltype(rb)::value, CB = decltype(cb)::value;
        const int64_t tiles = g.E * nt * ((g.M + 32 * WM * RB - 1) / (32 * WM * RB));
        const unsigned grid = (unsigned)((tiles + 7) / 8 * 8);
        if (g.prow) wgrad32_kernel<WM, WN, RB, CB, 1><<<grid, THREADS, 0, s>>>(g);
        else if (g.qrow) wgrad32_kernel<WM, WN, RB, CB, 2><<<grid, THREADS, 0, s>>>(g);
        else wgrad32_kernel<WM, WN, RB, CB, 0><<<grid, THREADS, 0, s>>>(g);
    });
    return hipGetLastError();
}

}  // namespace emu
