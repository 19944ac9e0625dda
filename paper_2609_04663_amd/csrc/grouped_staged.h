// The grouped products staged through registers: FP32 operands, split into their
// BF16 components on the way (six component products, Eq. fp32six), and 16-bit
// operands whose rows do not start on 16 bytes (the others: grouped16.h).
//
// A workgroup of eight waves computes a tile of 256 x 128 (or of 192 or 128 rows),
// a k-block (32 indices of FP32, 64 of 16 bits) at a time.  The entries of the
// k-block after the next are loaded into registers (24 or 48 of a lane); FP32 is split there
// (v_cvt_pk_bf16_f32, an exact subtraction; five instructions an entry); they are
// written to the LDS stage that the k-block before has released: every entry is
// split once for the whole tile, nothing goes through memory, and gathered
// rows, strides and odd extents cost nothing extra.  Two waves share a SIMD
// (waves w and w + 4): the one splits and writes while the other's matrix
// instructions run, then they change over; a k-block is one barrier.
//
// FP32 accumulates A0B0 in one set of registers and the five smaller products in
// another, added at the end.  Unlike the library's SGEMM the leading product is not
// flushed per panel of 256: 16 exact products are added per rounding, so even at
// K = 8192 the 512 roundings of a sum stay below those of a plain FP32 product.
//
// Bytes in LDS per k-block of FP32 at 256 x 128: 74 KB written, 196 KB read while
// its MFMAs take 3.1 thousand cycles, so the matrix instructions bound it: 8192 x 8192 x
// 8192 in one expert takes 5.1 to 5.7 ms (193 to 214 TFLOP/s), the library's SGEMM
// with its split pass 5.2.
#pragma once

#include "gemm_common.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

template <typename T>
using frag = T __attribute__((ext_vector_type(8)));
constexpr int BN = 128, THREADS = 512;

template <typename T>
struct Elem {
    using comp = T;                                   // what is staged in LDS
    static constexpr int PLANES = 1, BK = 64;
};
template <>
struct Elem<float> {
    using comp = bhalf;
    static constexpr int PLANES = 3, BK = 32;
};

__device__ __forceinline__ f32x16 mfma32(frag<bhalf> a, frag<bhalf> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(frag<half> a, frag<half> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// What loads of entries outside read: a row of zeros as wide as a tile.
__device__ __attribute__((aligned(16))) float g_zeros[256];

// Where chunk q (eight indices) of tile row r lies in a plane of a stage: the 16
// rows of a read phase touch 16 different 16-byte banks.
template <int BK>
__device__ __forceinline__ int chunk_at(int r, int q) {
    return r * (BK * 2) + ((q ^ (BK == 64 ? r >> 1 & 7 : swz(r))) << 4);
}

template <typename T>
__device__ __forceinline__ void put_chunk(char *dst, int plane, frag<T> x) {
    if constexpr (Elem<T>::PLANES == 1) {
        *reinterpret_cast<frag<T> *>(dst) = x;
    } else {
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const frag<bhalf> h = __builtin_convertvector(x, frag<bhalf>);
            *reinterpret_cast<frag<bhalf> *>(dst + c * plane) = h;
            if (c < 2) x = x - __builtin_convertvector(h, frag<float>);
        }
    }
}

// Whether this wave has its unit i of `units` units of a wave: a half one (192
// rows) is that of waves 0 to 3.
template <int UNITS_OF_ALL_WAVES>
__device__ __forceinline__ bool has_unit(int i) {
    return UNITS_OF_ALL_WAVES % 8 == 0 || i < UNITS_OF_ALL_WAVES / 8 ||
           __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < UNITS_OF_ALL_WAVES % 8;
}

// The loads of one operand, ROWS tile rows by the k-block, UNITS runs of eight
// indices to a thread.  Contiguous along the reduction: row(r) gives the stored
// row of tile row r, or -1 for zeros (row 0, which must exist, is read and not used).
template <typename T, int ROWS>
struct ContigLoads {
    static constexpr int BK = Elem<T>::BK, Q = BK / 8, ALL = ROWS * Q / 64, UNITS = (ALL + 7) / 8;
    frag<T> x[UNITS];
    const T *src[UNITS];
    bool there[UNITS];
    template <typename F>
    __device__ __forceinline__ void init(const T *base, int64_t ld, F row) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = threadIdx.x + THREADS * i;
            const int64_t r = has_unit<ALL>(i) ? row(u / Q) : -1;
            there[i] = r >= 0;
            src[i] = base + (there[i] ? r * ld : 0) + u % Q * 8;
        }
    }
    __device__ __forceinline__ void load(int k0, int K) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            if (!has_unit<ALL>(i)) continue;
            const T *const p = src[i] + k0;
            if (k0 + BK <= K) {
                x[i] = *reinterpret_cast<const vec<T, 8> *>(p);
            } else {
                const int left = K - k0 - (threadIdx.x + THREADS * i) % Q * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = j < left ? p[j] : T(0);
            }
        }
    }
    __device__ __forceinline__ void write(char *stage) const {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = threadIdx.x + THREADS * i;
            if (has_unit<ALL>(i)) put_chunk<T>(stage + chunk_at<BK>(u / Q, u % Q), ROWS * BK * 2, there[i] ? x[i] : frag<T>{});
        }
    }
};

// Contiguous along the tile rows (columns of W stored K x N; the operands of
// the matrix gradient): a wave takes 64 V tile rows of eight indices, a lane V
// of them (4 bytes), whose stored rows are uniform over the wave; look-ups in `map` are
// scalar loads.
template <typename T, int ROWS, bool MAP>
struct StridedLoads {
    static constexpr int BK = Elem<T>::BK, Q = BK / 8, V = 4 / sizeof(T);
    static constexpr int GROUPS = (ROWS + 64 * V - 1) / (64 * V), ALL = GROUPS * Q, UNITS = (ALL + 7) / 8;
    frag<T> x[UNITS][V];
    const T *base;
    unsigned ld, entries;
    const __attribute__((address_space(4))) int *map;
    unsigned col[UNITS];            // byte of the lane's first column
    int q[UNITS], r[UNITS], rows;
    __device__ __forceinline__ void init(const T *base_, int64_t ld_, const int *map_, int64_t entries_, int rows_) {
        base = base_;
        ld = (unsigned)ld_;
        map = (const __attribute__((address_space(4))) int *)map_;
        entries = MAP ? (unsigned)entries_ : 0xFFFFFFFFu;
        rows = rows_;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = wave + 8 * i;
            q[i] = u / GROUPS;
            r[i] = u % GROUPS * 64 * V + lane * V;
            // whole lanes of the tile: the others repeat its last ones
            col[i] = (r[i] + V <= rows ? r[i] : (rows >= V ? rows - V : 0)) * sizeof(T);
        }
    }
    // the lane's entries j of a row: 64-bit base in scalar registers, 32-bit offset
    __device__ __forceinline__ void at_row(const T *row, int i, int j) {
        asm volatile("" : "+s"(row));
        const char *const p = reinterpret_cast<const char *>(row) + col[i];
        if (V == 1 || rows >= V) {
            const vec<T, V> v = *reinterpret_cast<const vec<T, V> *>(p);
#pragma unroll
            for (int c = 0; c < V; ++c) x[i][c][j] = v[c];
        } else {
#pragma unroll
            for (int c = 0; c < V; ++c) x[i][c][j] = *reinterpret_cast<const T *>(p);      // one column
        }
    }
    __device__ __forceinline__ void load(int k0, int K) {
        if (MAP || k0 + BK > K) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                if (!has_unit<ALL>(i)) continue;
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
                    at_row(there ? base + (uint64_t)(unsigned)at[j] * ld : reinterpret_cast<const T *>(g_zeros), i, j);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                if (!has_unit<ALL>(i)) continue;
                const T *row = base + (uint64_t)(unsigned)(k0 + q[i] * 8) * ld;
#pragma unroll
                for (int j = 0; j < 8; ++j, row += ld) at_row(row, i, j);
            }
        }
    }
    __device__ __forceinline__ void write(char *stage) const {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            if (!has_unit<ALL>(i)) continue;
            // a lane that repeats the last columns writes them where they belong
            const int first = V == 1 ? r[i] : (int)(col[i] / sizeof(T));
#pragma unroll
            for (int c = 0; c < V; ++c)
                if (V == 1 || (first + c < ROWS && r[i] < ROWS))
                    put_chunk<T>(stage + chunk_at<BK>(first + c, q[i]), ROWS * BK * 2, x[i][c]);
        }
    }
};

// C = A B^T of the tile, rows x cols of it stored.  WM x WN waves of RB x CB
// blocks of 32 x 32.
template <typename T, int WM, int WN, int RB, int CB, typename A, typename B>
__device__ __forceinline__ void tile_product(A &a, B &b, int K, int rows, int cols, T *__restrict__ C,
                                             int64_t ldc, char *lds) {
    using comp = typename Elem<T>::comp;
    constexpr int PL = Elem<T>::PLANES, BK = Elem<T>::BK, RS = BK * 2;
    constexpr int AROWS = 32 * WM * RB, STAGE = PL * (AROWS + BN) * RS;
    static_assert(WM * WN == 8 && WN * CB * 32 == BN, "eight waves, 128 columns");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const bool early = wave < 4;
    f32x16 hi[RB][CB], lo[PL > 1 ? RB : 1][PL > 1 ? CB : 1];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            hi[i][j] = f32x16{};
            if constexpr (PL > 1) lo[i][j] = f32x16{};
        }
    if (K > 0) {
        a.load(0, K);
        b.load(0, K);
        a.write(lds);
        b.write(lds + PL * AROWS * RS);
        if (BK < K) {
            a.load(BK, K);
            b.load(BK, K);
        }
    }
    const int fa = wm * RB * 32 * RS, fb = PL * AROWS * RS + wn * CB * 32 * RS;
    int at = 0;
    for (int k0 = 0; k0 < K; k0 += BK) {
        __syncthreads();
        char *const cur = lds + at, *const nxt = lds + (STAGE - at);
        auto produce = [&]() __attribute__((always_inline)) {
            if (k0 + BK < K) {
                a.write(nxt);
                b.write(nxt + PL * AROWS * RS);
            }
            if (k0 + 2 * BK < K) {
                a.load(k0 + 2 * BK, K);
                b.load(k0 + 2 * BK, K);
            }
        };
        if (early) produce();
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            const int off = chunk_at<BK>(lane & 31, 2 * s + (lane >> 5));
            frag<comp> x[PL][RB], y[PL][CB];
#pragma unroll
            for (int c = 0; c < PL; ++c) {
#pragma unroll
                for (int i = 0; i < RB; ++i) 
                    x[c][i] = *reinterpret_cast<const frag<comp> *>(cur + fa + (c * AROWS + i * 32) * RS + off);
#pragma unroll
                for (int j = 0; j < CB; ++j) 
                    y[c][j] = *reinterpret_cast<const frag<comp> *>(cur + fb + (c * BN + j * 32) * RS + off);
            }
            // product-major: consecutive MFMAs write different accumulators
#pragma unroll
            for (int c = 0; c < PL; ++c)
#pragma unroll
                for (int d = 0; c + d < PL; ++d)
#pragma unroll
                    for (int i = 0; i < RB; ++i)
#pragma unroll
                        for (int j = 0; j < CB; ++j) {
                            if constexpr (PL > 1) {
                                if (c + d > 0) {
                                    lo[i][j] = mfma32(x[c][i], y[d][j], lo[i][j]);
                                    continue;
                                }
                            }
                            hi[i][j] = mfma32(x[c][i], y[d][j], hi[i][j]);
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
                float v = hi[i][j][r];
                if constexpr (PL > 1) v += lo[i][j][r];
                if (row < rows) C[row * ldc + col] = (T)v;
            }
        }
}

template <typename T, int AROWS>
constexpr int lds_bytes() { return 2 * Elem<T>::PLANES * (AROWS + BN) * Elem<T>::BK * 2; }

template <typename T, int WM, int WN, int RB, int CB, bool TB>
__global__ __launch_bounds__(THREADS, 2) void staged_gemm_kernel(GroupedGemm g) {
    constexpr int AROWS = 32 * WM * RB;
    __shared__ __attribute__((aligned(1024))) char lds[lds_bytes<T, AROWS>()];
    const RowTile t = RowTiles(g.offsets, g.E, g.R, AROWS, (g.N + BN - 1) / BN).of_workgroup(blockIdx.x);
    if (t.e < 0) return;
    const int rows = (int)(t.end - t.first), n0 = t.col * BN, cols = g.N - n0 < BN ? g.N - n0 : BN;
    // rows of no expert, or an X without rows: an empty reduction gives their zeros
    const bool none = t.e == g.E || g.xrows == 0;
    const T *const X = static_cast<const T *>(g.X);
    const T *const W = static_cast<const T *>(g.W) + (none ? 0 : t.e * g.sw);
    ContigLoads<T, AROWS> a;
    a.init(X, g.ldx, [&](int r) -> int64_t {
        const int64_t i = t.first + (r < rows ? r : rows - 1);
        if (!g.rows) return i;
        const int64_t m = g.rows[i];
        return m < g.xrows ? m : -1;
    });
    T *const C = static_cast<T *>(g.Y) + t.first * g.ldy + n0;
    const int K = none ? 0 : g.K;
    if constexpr (TB) {
        ContigLoads<T, BN> b;
        b.init(W + n0 * g.ldw, g.ldw, [&](int r) -> int64_t { return r < cols ? r : cols - 1; });
        tile_product<T, WM, WN, RB, CB>(a, b, K, rows, cols, C, g.ldy, lds);
    } else {
        StridedLoads<T, BN, false> b;
        b.init(W + n0, g.ldw, nullptr, 0, cols);
        tile_product<T, WM, WN, RB, CB>(a, b, K, rows, cols, C, g.ldy, lds);
    }
}

template <typename T, int WM, int WN, int RB, int CB, int MAPPED>  // the operand that goes through a map: 0 none, 1 P, 2 Q
__global__ __launch_bounds__(THREADS, 2) void staged_wgrad_kernel(GroupedWgrad g) {
    constexpr int AROWS = 32 * WM * RB;
    __shared__ __attribute__((aligned(1024))) char lds[lds_bytes<T, AROWS>()];
    const int mt = (g.M + AROWS - 1) / AROWS, nt = (g.N + BN - 1) / BN;
    // an XCD takes a contiguous run of tiles, so of (pieces of) experts
    const int64_t total = (int64_t)g.E * g.pieces * mt * nt, per = (total + 7) / 8;
    const int64_t id = blockIdx.x % 8 * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return;
    const int e = uniform(id / (mt * nt)), r = uniform(id % (mt * nt));
    const int m0 = r % mt * AROWS, n0 = r / mt * BN;
    const int rows = g.M - m0 < AROWS ? g.M - m0 : AROWS, cols = g.N - n0 < BN ? g.N - n0 : BN;
    int64_t lo, hi;
    expert_rows(g.offsets, g.E, g.R, e / g.pieces, lo, hi);
    piece_rows(e % g.pieces, g.pieces, lo, hi);
    lo = uniform(lo);
    const int K = uniform(hi - lo);
    StridedLoads<T, AROWS, MAPPED == 1> a;
    StridedLoads<T, BN, MAPPED == 2> b;
    a.init(static_cast<const T *>(g.P) + m0 + (MAPPED == 1 ? 0 : lo * g.ldp), g.ldp,
           MAPPED == 1 ? g.prow + lo : nullptr, g.prows, rows);
    b.init(static_cast<const T *>(g.Q) + n0 + (MAPPED == 2 ? 0 : lo * g.ldq), g.ldq,
           MAPPED == 2 ? g.qrow + lo : nullptr, g.qrows, cols);
    tile_product<T, WM, WN, RB, CB>(a, b, K, rows, cols, static_cast<T *>(g.dW) + e * g.sw + m0 * g.ldw + n0,
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

template <typename T>
hipError_t run_staged_gemm(const GroupedGemm &g, hipStream_t s) {
    const int64_t nt = (g.N + BN - 1) / BN;
    // an expert's last block is half full on average
    with_height(nt, [&](int h) { return (g.R + (int64_t)g.E * h / 2) / h; }, [&](auto wm, auto wn, auto rb, auto cb) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, RB = decltype(rb)::value, CB = decltype(cb)::value;
        const unsigned grid = (unsigned)((row_blocks_bound(g.R, g.E, 32 * WM * RB) * nt + 7) / 8 * 8);
        if (g.transb) staged_gemm_kernel<T, WM, WN, RB, CB, true><<<grid, THREADS, 0, s>>>(g);
        else staged_gemm_kernel<T, WM, WN, RB, CB, false><<<grid, THREADS, 0, s>>>(g);
    });
    return hipGetLastError();
}

template <typename T>
hipError_t run_staged_wgrad(const GroupedWgrad &g, hipStream_t s) {
    const int64_t nt = (g.N + BN - 1) / BN;
    with_height(nt * g.E * g.pieces, [&](int h) { return (g.M + h - 1) / h; }, [&](auto wm, auto wn, auto rb, auto cb) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, RB = decltype(rb)::value, CB = decltype(cb)::value;
        const int64_t tiles = g.E * g.pieces * nt * ((g.M + 32 * WM * RB - 1) / (32 * WM * RB));
        const unsigned grid = (unsigned)((tiles + 7) / 8 * 8);
        if (g.prow) staged_wgrad_kernel<T, WM, WN, RB, CB, 1><<<grid, THREADS, 0, s>>>(g);
        else if (g.qrow) staged_wgrad_kernel<T, WM, WN, RB, CB, 2><<<grid, THREADS, 0, s>>>(g);
        else staged_wgrad_kernel<T, WM, WN, RB, CB, 0><<<grid, THREADS, 0, s>>>(g);
    });
    return hipGetLastError();
}

}  // namespace emu
