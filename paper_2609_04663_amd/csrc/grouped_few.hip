// The grouped product for a few rows of each expert, bound by the bytes of the
// experts' matrices: every entry of W goes from memory to the registers of one
// wave, from there to the matrix instructions, and is not staged.
//
// v_mfma 16 x 16 x 32 with rows of X as rows and 16 columns of Y as columns.  A
// wave takes 64 columns (four tiles; one, if there are few) and 32 indices at a time:
//   W stored N x K: tile i is columns 16 i .. 16 i + 15, a lane loads eight
//     neighbouring indices of a column;
//   W stored K x N: a lane loads four neighbouring columns 4 l .. 4 l + 3 of eight
//     indices, and tile i is the columns 4 l + i: what a lane has loaded is what
//     the instructions want of it, with no exchange, and a row of 64 columns is
//     one run in memory.
// X lies in LDS (FP32 as three BF16 components, Eq. fp32split; W is split in
// registers), the 16-byte units of row t permuted by t % 16 so that the 16 rows of a
// read touch every bank once.  The waves of a workgroup share the reduction and
// add up their sums in LDS at the end, in order.  FP32 needs 150 to 190 registers, so
// a workgroup has four waves and three (two) of them share a CU; with eight only one
// did, and its start was in the open: 43 us for 32 rows over 32 experts of 1024 x 2048
// instead of 35.  16 bits need half of it and keep eight waves, which read longer runs
// of a row of W ('T': 105 us instead of 125 for 64 experts of 2048 x 2048, a row each).
//
// That case is 537 MB (5.2 TB/s), in FP32 1074 MB in 192 us (5.6 TB/s); loads alone
// reach 6.0 TB/s.
#include "emu_internal.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T>
using frag = T __attribute__((ext_vector_type(8)));

constexpr int STEP = 32;
constexpr int X_BYTES = 48 * 1024;          // of LDS, for X: room for two or three workgroups

template <typename T>
struct Elem {
    using comp = T;
    static constexpr int PLANES = 1, WAVES = 8;
};
template <>
struct Elem<float> {
    using comp = bhalf;
    static constexpr int PLANES = 3, WAVES = 4;
};

__device__ __forceinline__ f32x4 mfma16(frag<bhalf> a, frag<bhalf> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(frag<half> a, frag<half> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// The components of eight entries.
template <typename T>
__device__ __forceinline__ void components(const frag<T> &x, frag<typename Elem<T>::comp> (&c)[Elem<T>::PLANES]) {
    if constexpr (Elem<T>::PLANES == 1) {
        c[0] = x;
    } else {
        frag<float> r = x;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            c[i] = __builtin_convertvector(r, frag<bhalf>);
            if (i < 2) r = r - __builtin_convertvector(c[i], frag<float>);
        }
    }
}

// What a wave has loaded of W: 32 indices of its 16 NT columns.
template <typename T, int NT, bool TB>
struct Piece;
template <typename T, int NT>
struct Piece<T, NT, true> {
    frag<T> w[NT];
    // col: the lane's column of each tile; k: of its eight indices
    __device__ __forceinline__ void load(const T *W, int64_t ld, int col0, int N, int k0, int K, int lane) {
        const int k = k0 + 8 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int n = col0 + 16 * i + (lane & 15);
            const T *const p = W + (int64_t)(n < N ? n : N - 1) * ld + k;
            if (k0 + STEP <= K) {
                w[i] = *reinterpret_cast<const vec<T, 8> *>(p);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[i][j] = k + j < K ? p[j] : T(0);
            }
        }
    }
    __device__ __forceinline__ frag<T> tile(int i) const { return w[i]; }
    static __device__ __forceinline__ int column(int i, int c) { return 16 * i + c; }
};
template <typename T, int NT>
struct Piece<T, NT, false> {
    vec<T, NT> w[8];
    __device__ __forceinline__ void load(const T *W, int64_t ld, int col0, int N, int k0, int K, int lane) {
        const int k = k0 + 8 * (lane >> 4), n = col0 + NT * (lane & 15);
        if (k0 + STEP <= K && col0 + 16 * NT <= N) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const vec<T, NT> *>(W + (int64_t)(k + j) * ld + n);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    w[j][i] = k + j < K ? W[(int64_t)(k + j) * ld + (n + i < N ? n + i : N - 1)] : T(0);
        }
    }
    __device__ __forceinline__ frag<T> tile(int i) const {
        frag<T> f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = w[j][i];
        return f;
    }
    static __device__ __forceinline__ int column(int i, int c) { return NT * c + i; }
};

template <typename T, int MT, int NT, bool TB>
__global__ __launch_bounds__(64 * Elem<T>::WAVES, 2) void few_kernel(GroupedGemm g) {
    using C = typename Elem<T>::comp;
    constexpr int PL = Elem<T>::PLANES, WAVES = Elem<T>::WAVES, THREADS = 64 * WAVES, COLS = 16 * NT;
    __shared__ __attribute__((aligned(16))) char lds[X_BYTES];
    __shared__ float share[WAVES * MT * 256];
    __shared__ int row_of[16 * MT];
    const RowTile t = RowTiles(g.offsets, g.E, g.R, 16 * MT, (g.N + COLS - 1) / COLS).at(blockIdx.x);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4;
    const int m = (int)(t.end - t.first), K = g.K, N = g.N, col0 = t.col * COLS;
    T *const Y = static_cast<T *>(g.Y);
    if (t.e == g.E) {                                 // rows of no expert
        for (int i = threadIdx.x; i < m * COLS; i += THREADS)
            if (col0 + i % COLS < N) Y[(t.first + i / COLS) * g.ldy + col0 + i % COLS] = T(0.0f);
        return;
    }
    const T *const W = static_cast<const T *>(g.W) + t.e * g.sw;
    // steps of 32 indices: the waves take neighbouring ones; X for `chunk` of them at a time
    const int steps = (K + STEP - 1) / STEP, rounds = (steps + WAVES - 1) / WAVES;
    const int fit = X_BYTES / (PL * m * STEP * 2) / WAVES * WAVES;
    const int chunk = rounds * WAVES < fit ? rounds * WAVES : fit, RB = chunk * STEP * 2;
    const int in_chunk = chunk / WAVES;               // rounds
    if ((int)threadIdx.x < m) {
        const int64_t r = t.first + threadIdx.x, at = g.rows ? g.rows[r] : r;
        row_of[threadIdx.x] = at >= 0 && at < g.xrows ? (int)at : -1;
    }
    f32x4 hi[NT][MT] = {}, lo[PL > 1 ? NT : 1][PL > 1 ? MT : 1] = {};
    int at[MT];
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int tok = 16 * a + (lane & 15) < m ? 16 * a + (lane & 15) : m - 1;
        at[a] = tok;
    }
    // the 16-byte unit of row tok, plane c
    auto place = [&](int c, int tok, int unit) { return (c * m + tok) * RB + ((unit ^ (tok & 15)) << 4); };
    Piece<T, NT, TB> now, next;
    auto k_of = [&](int round) {
        const int s = round * WAVES + wave;
        return (s < steps ? s : steps - 1) * STEP;    // past the end: the last ones, not used
    };
    if (rounds > 0) now.load(W, g.ldw, col0, N, k_of(0), K, lane);
    __syncthreads();                                  // row_of
    for (int round = 0; round < rounds; ++round) {
        if (round % in_chunk == 0) {
            if (round > 0) __syncthreads();           // every wave is done with the chunk before
            const int k0 = round * WAVES * STEP, units = chunk * STEP / 8;
            for (int u = threadIdx.x; u < m * units; u += THREADS) {
                const int tok = u / units, unit = u % units, k = k0 + unit * 8;
                frag<T> x = frag<T>{};
                if (row_of[tok] >= 0 && k < K) {
                    const T *const p = static_cast<const T *>(g.X) + row_of[tok] * g.ldx + k;
                    if (k + 8 <= K) {
                        x = *reinterpret_cast<const vec<T, 8> *>(p);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[j] = k + j < K ? p[j] : T(0);
                    }
                }
                frag<C> c[PL];
                components<T>(x, c);
#pragma unroll
                for (int i = 0; i < PL; ++i) *reinterpret_cast<frag<C> *>(lds + place(i, tok, unit)) = c[i];
            }
            __syncthreads();
        }
        next.load(W, g.ldw, col0, N, k_of(round + 1 < rounds ? round + 1 : round), K, lane);
        if (round * WAVES + wave < steps) {
            const int unit = (round % in_chunk * WAVES + wave) * (STEP / 8) + h;
            frag<C> x[MT][PL];
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int c = 0; c < PL; ++c) x[a][c] = *reinterpret_cast<const frag<C> *>(lds + place(c, at[a], unit));
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                frag<C> w[PL];
                components<T>(now.tile(i), w);
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    hi[i][a] = mfma16(x[a][0], w[0], hi[i][a]);
                    if constexpr (PL > 1) {
#pragma unroll
                        for (int s = 2; s > 0; --s)   // A_c B_d with c + d = 2, then 1
#pragma unroll
                            for (int c = 0; c <= s; ++c) lo[i][a] = mfma16(x[a][c], w[s - c], lo[i][a]);
                    }
                }
            }
        }
        now = next;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = hi[i][a][r];
                if constexpr (PL > 1) v += lo[i][a][r];
                share[(wave * MT + a) * 256 + (4 * h + r) * 16 + (lane & 15)] = v;
            }
        __syncthreads();
        for (int j = threadIdx.x; j < m * 16; j += THREADS) {
            const int tok = j / 16, c = j % 16, col = col0 + Piece<T, NT, TB>::column(i, c);
            if (col >= N) continue;
            float v = 0.0f;
            for (int w = 0; w < WAVES; ++w) v += share[(w * MT + tok / 16) * 256 + tok % 16 * 16 + c];
            Y[(t.first + tok) * g.ldy + col] = (T)v;
        }
    }
}

}  // namespace

hipError_t launch_few(const GroupedGemm &g, hipStream_t s) {
    using std::integral_constant;
    const int mt = g.R <= 16 * (int64_t)g.E ? 1 : 2;
    auto tiles = [&](int nt) { return row_blocks_bound(g.R, g.E, 16 * mt) * ((g.N + 16 * nt - 1) / (16 * nt)); };
    // 16 columns instead of 64 where the tiles would not fill the chip: 4096 x 4096, one
    // row, 'T': 16 bits 19 -> 9.7 us, float32 42 -> 22; 'N', 16 rows, float32 58 -> 43.
    // Not for 16 bits 'N', whose loads are then runs of 32 bytes: 8 rows 18 -> 24.
    const int nt = tiles(4) < device_cu_count() && (g.transb || g.dtype == EMU_F32) ? 1 : 4;
    with_type(g.dtype, [&](auto z) {
        using T = decltype(z);
        constexpr bool F32 = std::is_same<T, float>::value;
        auto run = [&](auto m, auto n, auto tb) {
            constexpr int MT = decltype(m)::value, NT = decltype(n)::value, THREADS = 64 * Elem<T>::WAVES;
            few_kernel<T, MT, NT, decltype(tb)::value><<<(unsigned)tiles(NT), THREADS, 0, s>>>(g);
        };
        const integral_constant<int, 1> one;
        const integral_constant<int, 2> two;
        const integral_constant<int, 4> four;
        auto columns = [&](auto m, auto tb) {
            if constexpr (F32 || decltype(tb)::value)
                if (nt == 1) return run(m, one, tb);
            run(m, four, tb);
        };
        auto layout = [&](auto tb) {
            // 16 bits 'T' come here with 8 rows of each expert at most
            if constexpr (F32 || !decltype(tb)::value)
                if (mt == 2) return columns(two, tb);
            columns(one, tb);
        };
        if (g.transb) layout(std::true_type{});
        else layout(std::false_type{});
    });
    return hipGetLastError();
}

}  // namespace emu
