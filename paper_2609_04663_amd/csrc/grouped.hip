// Products of rows with the matrix of each row's expert, and the gradient of
// those matrices, for rows ordered by expert with any number of rows each.
//
//   emu_grouped_gemm    Y[r] = X[r] W[e(r)]            (W as K x N or N x K)
//   emu_grouped_wgrad   dW[e] = sum of P[r]^T Q[r] over the rows r of e
//
// Elements.  bfloat16 and half products are exact in FP32 and accumulated there
// by the 32 x 32 x 16 MFMA, rounded once at the end.  FP32 operands are split
// into three BF16 components each where they are staged (Eq. fp32split), and
// the six products A_i B_j, i + j < 3 (Eq. fp32six), go to two FP32 accumulator
// sets: A0B0 to one, the five smaller products to the other, added at the end.
// Unlike the library's SGEMM the leading product is not flushed per panel of
// 256: 16 exact products are added per rounding, so even at K = 8192 the 512
// roundings of a sum stay below those of a plain FP32 product, and the 64
// registers of a third set buy the second workgroup of a CU.
//
// Layout.  A workgroup of four waves computes a tile of BM rows by 128 columns,
// one k-block (32 indices of FP32, 64 of the others) at a time: global memory to
// registers (the k-block ahead), registers to LDS, fragments to the MFMA.  A row
// of a k-block is K-contiguous in LDS, 16 bytes longer than its data, so that the
// 16 lanes of a read or write phase touch 16 different 16-byte banks.  An
// operand that is contiguous along the other direction (W stored K x N; both
// operands of the matrix gradient) is transposed in registers: a lane takes two
// columns by eight indices.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
template <typename T>
using frag = T __attribute__((ext_vector_type(8)));

constexpr int BN = 128, THREADS = 256;
constexpr int64_t OFFSETS = (int64_t)1 << 31;        // leading dimensions that the FP32 kernels take

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

// Eight entries along the reduction, as loaded, to the planes of a stage.
template <typename T>
struct Put {
    static __device__ __forceinline__ void to(char *dst, int, const frag<T> &x) {
        *reinterpret_cast<frag<T> *>(dst) = x;
    }
};
template <>
struct Put<float> {
    static __device__ __forceinline__ void to(char *dst, int plane, const frag<float> &x) {
        frag<float> r = x;
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const frag<bhalf> h = __builtin_convertvector(r, frag<bhalf>);
            *reinterpret_cast<frag<bhalf> *>(dst + c * plane) = h;
            if (c < 2) r = r - __builtin_convertvector(h, frag<float>);
        }
    }
};

// One operand of a tile: ROWS tile rows by the reduction.  Contiguous along the
// reduction: element (row, k) at base + index(row) ld + k.  Strided: at
// base + index(k) ld + row.  index is the number itself or a look-up in `map`,
// whose entries outside [0, entries) stand for rows of zeros.
template <typename T>
struct Operand {
    const T *base;
    int64_t ld;
    const int *map;
    int64_t entries;
    int64_t rows;           // tile rows that exist
};

template <typename T, int ROWS, bool CONTIG>
struct Stager;

template <typename T, int ROWS>
struct Stager<T, ROWS, true> {
    static constexpr int BK = Elem<T>::BK, Q = BK / 8, RS = BK * 2 + 16;
    static constexpr int UNITS = (ROWS * Q + THREADS - 1) / THREADS;
    frag<T> x[UNITS];
    const T *src[UNITS];
    bool there[UNITS];
    // unit i of a thread: tile row (tid + THREADS i) / Q, indices 8 ((tid + ...) % Q)
    __device__ __forceinline__ void init(const Operand<T> &o) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int64_t row = (threadIdx.x + THREADS * i) / Q;
            int64_t at = row < o.rows ? row : o.rows - 1;
            there[i] = true;
            if (o.map) {
                at = o.map[at];
                there[i] = at >= 0 && at < o.entries;
                if (!there[i]) at = 0;
            }
            src[i] = o.base + at * o.ld;
        }
    }
    __device__ __forceinline__ void load(const Operand<T> &, int64_t k0, int64_t K) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int64_t k = k0 + (threadIdx.x + THREADS * i) % Q * 8;
            if (k0 + BK <= K) {
                x[i] = *reinterpret_cast<const vec<T, 8> *>(src[i] + k);
                if (!there[i]) x[i] = frag<T>{};
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[i][j] = there[i] && k + j < K ? src[i][k + j] : T(0);
            }
        }
    }
    __device__ __forceinline__ void store(char *lds) const {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = threadIdx.x + THREADS * i;
            if (ROWS * Q % THREADS == 0 || u < ROWS * Q)
                Put<T>::to(lds + u / Q * RS + u % Q * 16, ROWS * RS, x[i]);
        }
    }
};

template <typename T, int ROWS>
struct Stager<T, ROWS, false> {
    static constexpr int BK = Elem<T>::BK, Q = BK / 8, RS = BK * 2 + 16;
    static constexpr int UNITS = ROWS / 2 * Q / THREADS;
    static_assert(ROWS == 128 && UNITS * THREADS == ROWS / 2 * Q, "whole waves");
    frag<T> x[UNITS][2];
    __device__ __forceinline__ void init(const Operand<T> &) {}
    // unit i: columns 2 lane, 2 lane + 1 of the indices 8 (wave + 4 i) ..
    __device__ __forceinline__ void load(const Operand<T> &o, int64_t k0, int64_t K) {
        const int c = (threadIdx.x & 63) * 2;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t k = k0 + (wave + 4 * i) * 8 + j;
                int64_t at = k;
                bool there = k < K;
                if (o.map && there) {
                    at = o.map[k];
                    there = at >= 0 && at < o.entries;
                }
                const T *const p = o.base + (there ? at : 0) * o.ld;
                if (!there) {
                    x[i][0][j] = x[i][1][j] = T(0);
                } else if (o.rows >= ROWS) {
                    const vec<T, 2> v = *reinterpret_cast<const vec<T, 2> *>(p + c);
                    x[i][0][j] = v[0];
                    x[i][1][j] = v[1];
                } else {
                    x[i][0][j] = p[c < o.rows ? c : o.rows - 1];
                    x[i][1][j] = p[c + 1 < o.rows ? c + 1 : o.rows - 1];
                }
            }
    }
    __device__ __forceinline__ void store(char *lds) const {
        const int c = (threadIdx.x & 63) * 2, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                Put<T>::to(lds + (c + j) * RS + (wave + 4 * i) * 16, ROWS * RS, x[i][j]);
    }
};

// C (a.rows x b.rows, at most BM x 128) = A B^T over k in [0, K) of the two
// operands' reductions.
template <typename T, int BM, bool CA, bool CB>
__device__ __forceinline__ void tile_product(const Operand<T> &a, const Operand<T> &b, int64_t K,
                                             T *__restrict__ C, int64_t ldc, char *lds) {
    using comp = typename Elem<T>::comp;
    constexpr int PL = Elem<T>::PLANES, BK = Elem<T>::BK, RS = BK * 2 + 16;
    constexpr int WM = BM >= 64 ? 2 : 1, WN = 4 / WM;          // waves along the rows, the columns
    constexpr int RB = BM / 32 / WM, CBK = BN / 32 / WN;       // 32 x 32 blocks of a wave
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    char *const la = lds, *const lb = lds + PL * BM * RS;
    f32x16 hi[RB][CBK], lo[PL > 1 ? RB : 1][PL > 1 ? CBK : 1];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CBK; ++j) {
            hi[i][j] = f32x16{};
            if constexpr (PL > 1) lo[i][j] = f32x16{};
        }
    Stager<T, BM, CA> sa;
    Stager<T, BN, CB> sb;
    sa.init(a);
    sb.init(b);
    if (K > 0) {
        sa.load(a, 0, K);
        sb.load(b, 0, K);
    }
    const int fa = (wm * RB * 32 + (lane & 31)) * RS + (lane >> 5) * 16;
    const int fb = (wn * CBK * 32 + (lane & 31)) * RS + (lane >> 5) * 16;
    for (int64_t k0 = 0; k0 < K; k0 += BK) {
        __syncthreads();
        sa.store(la);
        sb.store(lb);
        __syncthreads();
        if (k0 + BK < K) {
            sa.load(a, k0 + BK, K);
            sb.load(b, k0 + BK, K);
        }
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            frag<comp> x[PL][RB], y[PL][CBK];
#pragma unroll
            for (int c = 0; c < PL; ++c) {
#pragma unroll
                for (int i = 0; i < RB; ++i)
                    x[c][i] = *reinterpret_cast<const frag<comp> *>(la + (c * BM + i * 32) * RS + fa + s * 32);
#pragma unroll
                for (int j = 0; j < CBK; ++j)
                    y[c][j] = *reinterpret_cast<const frag<comp> *>(lb + (c * BN + j * 32) * RS + fb + s * 32);
            }
            // product-major: consecutive MFMAs write different accumulators
#pragma unroll
            for (int c = 0; c < PL; ++c)
#pragma unroll
                for (int d = 0; c + d < PL; ++d)
#pragma unroll
                    for (int i = 0; i < RB; ++i)
#pragma unroll
                        for (int j = 0; j < CBK; ++j) {
                            if constexpr (PL > 1) {
                                if (c + d > 0) {
                                    lo[i][j] = mfma32(x[c][i], y[d][j], lo[i][j]);
                                    continue;
                                }
                            }
                            hi[i][j] = mfma32(x[c][i], y[d][j], hi[i][j]);
                        }
        }
    }
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CBK; ++j) {
            const int64_t col = (wn * CBK + j) * 32 + (lane & 31);
            if (col >= b.rows) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // accumulator register r of a lane: row 8 (r / 4) + r % 4 + 4 (lane / 32)
                const int64_t row = (wm * RB + i) * 32 + (r >> 2) * 8 + (r & 3) + (lane >> 5) * 4;
                if (row >= a.rows) continue;
                float v = hi[i][j][r];
                if constexpr (PL > 1) v += lo[i][j][r];
                C[row * ldc + col] = (T)v;
            }
        }
}

template <typename T, int BM>
constexpr int stage_bytes() {
    return Elem<T>::PLANES * (BM + BN) * (Elem<T>::BK * 2 + 16);
}

template <typename T, int BM, bool CB>
__global__ __launch_bounds__(THREADS, 2) void grouped_gemm_kernel(
    const T *__restrict__ X, int64_t ldx, int64_t xrows, const int *__restrict__ rows,
    const T *__restrict__ W, int64_t ldw, int64_t sw, const int *__restrict__ offsets, int E, int64_t R,
    T *__restrict__ Y, int64_t ldy, int N, int K) {
    __shared__ __attribute__((aligned(16))) char lds[stage_bytes<T, BM>()];
    const RowTile t = RowTiles(offsets, E, R, BM, (N + BN - 1) / BN).of_workgroup(blockIdx.x);
    if (t.e < 0) return;
    const int64_t n0 = (int64_t)t.col * BN;
    T *const C = Y + t.first * ldy + n0;
    const int64_t cols = N - n0 < BN ? N - n0 : BN;
    Operand<T> a = {X + (rows ? 0 : t.first * ldx), ldx, rows ? rows + t.first : nullptr, xrows,
                    t.end - t.first};
    // rows of no expert: an empty reduction gives their zeros
    const bool none = t.e == E;
    const T *const We = W + (none ? 0 : t.e * sw);
    Operand<T> b = {CB ? We + n0 * ldw : We + n0, ldw, nullptr, 0, cols};
    tile_product<T, BM, true, CB>(a, b, none ? 0 : K, C, ldy, lds);
}

template <typename T>
__global__ __launch_bounds__(THREADS, 2) void grouped_wgrad_kernel(
    const T *__restrict__ P, int64_t ldp, int64_t prows, const int *__restrict__ prow,
    const T *__restrict__ Q, int64_t ldq, int64_t qrows, const int *__restrict__ qrow,
    const int *__restrict__ offsets, int E, int64_t R, T *__restrict__ dW, int64_t ldw, int64_t sw,
    int M, int N) {
    constexpr int BM = 128;
    __shared__ __attribute__((aligned(16))) char lds[stage_bytes<T, BM>()];
    const int mt = (M + BM - 1) / BM, nt = (N + BN - 1) / BN;
    const int64_t id = blockIdx.x;
    const int e = (int)(id / (mt * nt)), r = (int)(id % (mt * nt));
    const int64_t m0 = (int64_t)(r % mt) * BM, n0 = (int64_t)(r / mt) * BN;
    int64_t lo, hi;
    expert_rows(offsets, E, R, e, lo, hi);
    Operand<T> a = {P + m0 + (prow ? 0 : lo * ldp), ldp, prow ? prow + lo : nullptr, prows,
                    M - m0 < BM ? M - m0 : BM};
    Operand<T> b = {Q + n0 + (qrow ? 0 : lo * ldq), ldq, qrow ? qrow + lo : nullptr, qrows,
                    N - n0 < BN ? N - n0 : BN};
    tile_product<T, BM, false, false>(a, b, hi - lo, dW + e * sw + m0 * ldw + n0, ldw, lds);
}

}  // namespace

hipError_t launch_grouped_gemm(const GroupedGemm &g, hipStream_t s) {
    if (direct_gemm(g) && g.R > 32 * (int64_t)g.E)
        return launch_direct_gemm(g, g.R >= 512 * (int64_t)g.E ? 256 : 128, s);
    if (g.dtype == EMU_F32 && g.R >= 64 * (int64_t)g.E && g.ldw < OFFSETS) return launch_gemm32(g, s);
    auto run = [&](auto z, auto bm, auto cb) {
        using T = decltype(z);
        constexpr int BM = decltype(bm)::value;
        const int64_t tiles = row_blocks_bound(g.R, g.E, BM) * ((g.N + BN - 1) / BN);
        grouped_gemm_kernel<T, BM, decltype(cb)::value><<<(unsigned)((tiles + 7) / 8 * 8), THREADS, 0, s>>>(
            static_cast<const T *>(g.X), g.ldx, g.xrows, g.rows, static_cast<const T *>(g.W), g.ldw,
            g.sw, g.offsets, g.E, g.R, static_cast<T *>(g.Y), g.ldy, g.N, g.K);
    };
    with_type(g.dtype, [&](auto z) {
        auto layout = [&](auto bm) {
            if (g.transb) run(z, bm, std::true_type{});
            else run(z, bm, std::false_type{});
        };
        if (g.R <= 32 * (int64_t)g.E) layout(std::integral_constant<int, 32>{});
        else layout(std::integral_constant<int, 128>{});
    });
    return hipGetLastError();
}

hipError_t launch_grouped_wgrad(const GroupedWgrad &g, hipStream_t s) {
    if (direct_wgrad(g)) return launch_direct_wgrad(g, g.M >= 512 && g.N >= 512 ? 256 : 128, s);
    if (g.dtype == EMU_F32 && g.ldp < OFFSETS && g.ldq < OFFSETS) return launch_wgrad32(g, s);
    const int64_t tiles = (int64_t)g.E * ((g.M + 127) / 128) * ((g.N + BN - 1) / BN);
    with_type(g.dtype, [&](auto z) {
        using T = decltype(z);
        grouped_wgrad_kernel<T><<<(unsigned)tiles, THREADS, 0, s>>>(
            static_cast<const T *>(g.P), g.ldp, g.prows, g.prow, static_cast<const T *>(g.Q), g.ldq,
            g.qrows, g.qrow, g.offsets, g.E, g.R, static_cast<T *>(g.dW), g.ldw, g.sw, g.M, g.N);
    });
    return hipGetLastError();
}

}  // namespace emu
