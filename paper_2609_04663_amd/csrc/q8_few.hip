// The product of 8-bit integers for a few rows of each expert, bound by the bytes of the
// experts' matrices: every entry of W and X goes from memory to the registers of one wave
// and from there to the matrix instructions.  Any alignment.
//
// v_mfma 16 x 16 x 64 with rows of X as rows and 16 columns of Y as columns.  A wave
// takes 16 NT columns and 128 indices at a time: a lane loads 16 neighbouring indices of
// its row or column twice, 64 apart.  The waves of a workgroup take neighbouring runs of
// 128 and add up their 32-bit sums in LDS at the end.
//
// One row of 4096 x 4096 takes 6.0 us (2.8 TB/s; a launch, and four rounds of loads that wait for
// one another), 8 rows over 64 experts of 2048 x 2048 9.8 with the call.  Six rounds in flight
// instead of two spilled and lost where they were tried (16 rows of 8192 x 8192 in 16 columns 18.1
// and 19.4 us); one row alone, which holds 67 of its 128 registers, was not.
#include "emu_internal.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int STEP = 128, WAVES = Q8_FEW_ROUND / STEP, THREADS = 64 * WAVES;

__device__ __forceinline__ i32x4 mfma16(i32x4 a, i32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// The N rows of a lane.  SHIFT: not all of them at multiples of 4, where a 16-byte load of
// its own address takes two to three times as long: five whole words around the bytes are
// read, and moved when they are used.  Not in a matrix's first and last rows, whose
// words may lie partly outside of it.  16 rows of 16384 x 8192 at odd addresses: 34 us, with
// the loads of their own addresses 73; 60 of 4096 x 4095 20 and 31.
template <int N, bool SHIFT>
struct Rows {
    const int8_t *at[N];
    int by[N];                      // bytes that at[i] lies before the row
    __device__ __forceinline__ void set(int i, const int8_t *row, bool edge) {
        by[i] = SHIFT && !edge ? (int)((uintptr_t)row & 3) : 0;
        at[i] = row - by[i];
    }
};
template <int N, bool SHIFT>
struct Piece {                      // 128 indices of N rows of a lane
    i32x4 v[N][2];
    int last[SHIFT ? N : 1][2];
    __device__ __forceinline__ void load(const Rows<N, SHIFT> &row, int k0, int K, int h) {
        typedef int __attribute__((ext_vector_type(4), aligned(1))) unaligned;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int k = k0 + 64 * p + 16 * h;
                if (k0 + STEP <= K) {
                    v[i][p] = *reinterpret_cast<const unaligned *>(row.at[i] + k);
                    if constexpr (SHIFT)
                        last[i][p] = row.by[i] > 0 ? *reinterpret_cast<const int *>(row.at[i] + k + 16) : 0;
                } else {
                    v[i][p] = load_bytes16(row.at[i] + row.by[i], k, K);
                }
            }
    }
    // whole: of a step that the row does not end in
    __device__ __forceinline__ i32x4 get(const Rows<N, SHIFT> &row, int i, int p, bool whole) const {
        if constexpr (!SHIFT) return v[i][p];
        const int by = whole ? row.by[i] : 0;
        i32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int next = j < 3 ? v[i][p][(j + 1) % 4] : last[SHIFT ? i : 0][p];
            r[j] = (int)__builtin_amdgcn_alignbyte((unsigned)next, (unsigned)v[i][p][j], by);
        }
        return r;
    }
};

// One tile; share: the waves' sums.
template <typename T, int MT, int NT, bool SHIFT>
__device__ __forceinline__ void q8_few_tile(const Q8Gemm &g, const RowTile &t, int (&share)[WAVES][MT][NT][256]) {
    constexpr int COLS = 16 * NT;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4;
    const int m = (int)(t.end - t.first), K = g.K, N = g.N, col0 = t.col * COLS;
    T *const Y = static_cast<T *>(g.Y) + t.first * g.ldy + col0;
    if (t.e == g.E) {                                 // rows of no expert
        for (int i = threadIdx.x; i < m * COLS; i += THREADS)
            if (col0 + i % COLS < N) Y[i / COLS * g.ldy + i % COLS] = T(0.0f);
        return;
    }
    const int steps = (K + STEP - 1) / STEP, rounds = (steps + WAVES - 1) / WAVES;
    Rows<MT, SHIFT> xrow;
    Rows<NT, SHIFT> wrow;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int col = col0 + 16 * i + (lane & 15), n = col < N ? col : N - 1;
        wrow.set(i, g.W + t.e * g.sw + n * g.ldw, n == 0 || n == N - 1);
    }
#pragma unroll
    for (int a = 0; a < MT; ++a) {                    // rows past the last repeat it, ones outside X row 0
        const int r = 16 * a + (lane & 15);
        int64_t at = t.first + (r < m ? r : m - 1);
        if (g.rows) at = g.rows[at];
        at = at >= 0 && at < g.xrows ? at : 0;
        xrow.set(a, g.X + at * g.ldx, at == 0 || at == g.xrows - 1);
    }
    i32x4 acc[MT][NT] = {};
    Piece<NT, SHIFT> w, w_next;
    Piece<MT, SHIFT> x, x_next;
    auto k_of = [&](int round) {
        const int s = round * WAVES + wave;
        return (s < steps ? s : steps - 1) * STEP;    // past the end: the last ones, not used
    };
    const bool any = rounds > 0 && g.xrows > 0;       // else there is nothing to read
    if (any) {
        w_next.load(wrow, k_of(0), K, h);
        x_next.load(xrow, k_of(0), K, h);
    }
    for (int round = 0; any && round < rounds; ++round) {
        w = w_next;
        x = x_next;
        if (round + 1 < rounds) {
            w_next.load(wrow, k_of(round + 1), K, h);
            x_next.load(xrow, k_of(round + 1), K, h);
        }
        if (round * WAVES + wave < steps) {
            const bool whole = k_of(round) + STEP <= K;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                i32x4 f[MT];
#pragma unroll
                for (int a = 0; a < MT; ++a) f[a] = x.get(xrow, a, p, whole);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const i32x4 c = w.get(wrow, i, p, whole);
#pragma unroll
                    for (int a = 0; a < MT; ++a) acc[a][i] = mfma16(f[a], c, acc[a][i]);
                }
            }
        }
    }
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) share[wave][a][i][(4 * h + r) * 16 + (lane & 15)] = acc[a][i][r];
    __syncthreads();
    for (int j = threadIdx.x; j < m * COLS; j += THREADS) {
        const int r = j / COLS, c = j % COLS;
        if (col0 + c >= N) continue;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += share[w][r / 16][c / 16][r % 16 * 16 + c % 16];
        if constexpr (std::is_same<T, int>::value) {
            Y[r * g.ldy + c] = sum;
        } else {
            const int64_t at = g.rows ? g.rows[t.first + r] : t.first + r;
            const bool there = at >= 0 && at < g.xrows;   // zeros for a row outside X, whatever W's scale
            Y[r * g.ldy + c] = (T)(there ? q8_result(sum, g.ws[(int64_t)t.e * N + col0 + c], g.xs[at]) : 0.0f);
        }
    }
}

// Workgroups to a CU, by the registers that the kernel needs.  With four sets of one kind and one
// of the other, two workgroups spill 5 to 8: one to a CU without spills takes 23.5 us instead of
// 24.8 for 16 rows of 16384 x 8192 in 64 columns, but 26.0 instead of 23.8 for 64 of 8192 x 4096 in
// 16, 43 instead of 40 for 64 of 8192 x 8192.
constexpr int few_per_cu(int mt, int nt, bool shift) { return mt + nt >= (shift ? 4 : 6) ? 1 : 2; }

// T int: the sums of a split.
template <typename T, int MT, int NT, bool SHIFT>
__global__ __launch_bounds__(THREADS, 2 * few_per_cu(MT, NT, SHIFT)) void q8_few_kernel(Q8Gemm g) {
    constexpr int COLS = 16 * NT;
    __shared__ int share[WAVES][MT][NT][256];
    if constexpr (std::is_same<T, int>::value) to_split(g);
    const RowTiles tiles(g.offsets, g.E, g.R, 16 * MT, (g.N + COLS - 1) / COLS);
    for (int64_t id = blockIdx.x;; id += gridDim.x) {
        const RowTile t = tiles.at(id);
        if (t.e < 0) return;
        q8_few_tile<T, MT, NT, SHIFT>(g, t, share);
        __syncthreads();                              // every sum has been read
    }
}

}  // namespace

// Rows and columns of a tile, in sixteens: rows for those of an expert on average, 64 at most;
// as many columns as fill the chip.  Calls with 16, 32 and 64 columns: 16 rows of 8192 x 4096 10.5, 9.0
// and 12.8 us, of 16384 x 8192 31.5, 32.9 and 24.8; 32 rows of 8192 x 4096 14.1, 10.7 and 14.8, of 8192 x
// 8192 24.4, 21.9 and 25.0; 64 rows of 8192 x 4096 23.8, 16.3 and 19.8.  At 8192 x 8192 the rule's
// 32 columns are not the best for 16 rows (18.0, 20.5 and 21.4) or one (14.3, 19.8 and 18.5).
static int row_sets(const Q8Gemm &g) {
    return g.R <= 16 * (int64_t)g.E ? 1 : (g.R <= 32 * (int64_t)g.E ? 2 : 4);
}
static int64_t expected(const Q8Gemm &g, int nt) {
    return row_blocks_expected(g.R, g.E, 16 * row_sets(g)) * ((g.N + 16 * nt - 1) / (16 * nt));
}
static bool in_words(const Q8Gemm &g) {
    return ((reinterpret_cast<uintptr_t>(g.X) | reinterpret_cast<uintptr_t>(g.W) | g.ldx | g.ldw | g.sw) & 3) == 0;
}
// (Rows that are moved take more registers: with 64 columns one workgroup has a CU; 854 rows over 64
// experts of 1280 x 1081 73 us instead of 66.)
static int column_sets(const Q8Gemm &g) {
    const int64_t cus = device_cu_count();
    return expected(g, 4) >= cus && in_words(g) ? 4 : (expected(g, 2) >= cus ? 2 : 1);
}

Q8FewShape q8_few_shape(const Q8Gemm &g) {
    const int mt = row_sets(g), nt = column_sets(g);
    return {(double)expected(g, nt), mt, nt, few_per_cu(mt, nt, !in_words(g)), in_words(g)};
}

template <typename T>
static void launch(const Q8Gemm &g, int splits, hipStream_t s) {
    using std::integral_constant;
    // (no expert: rows of zeros)
    const int mt = g.E > 0 ? row_sets(g) : 4, nt = g.E > 0 ? column_sets(g) : 4;
    auto tiles = [&](int nt) { return row_blocks_bound(g.R, g.E, 16 * mt) * ((g.N + 16 * nt - 1) / (16 * nt)); };
    const bool shift = !in_words(g);
    auto run = [&](auto m, auto n) {
        constexpr int MT = decltype(m)::value, NT = decltype(n)::value;
        const int64_t most = (1 << 22) / splits;
        const dim3 grid((unsigned)(tiles(NT) < most ? tiles(NT) : most), splits);
        if constexpr (NT < 4)
            if (shift) return q8_few_kernel<T, MT, NT, true><<<grid, THREADS, 0, s>>>(g);
        q8_few_kernel<T, MT, NT, false><<<grid, THREADS, 0, s>>>(g);
    };
    auto columns = [&](auto m) {
        if constexpr (std::is_same<T, int>::value) {
            run(m, integral_constant<int, 1>{});        // splits are of few columns
        } else {
            if (nt == 1) run(m, integral_constant<int, 1>{});
            else if (nt == 2) run(m, integral_constant<int, 2>{});
            else run(m, integral_constant<int, 4>{});
        }
    };
    if (mt == 1) columns(integral_constant<int, 1>{});
    else if (mt == 2) columns(integral_constant<int, 2>{});
    else columns(integral_constant<int, 4>{});
}

hipError_t launch_q8_few(const Q8Gemm &g, hipStream_t s) {
    with_type(g.dtype, [&](auto z) { launch<decltype(z)>(g, 1, s); });
    return hipGetLastError();
}
hipError_t launch_q8_few_sums(const Q8Gemm &g, int splits, hipStream_t s) {
    launch<int>(g, splits, s);
    return hipGetLastError();
}

}  // namespace emu
