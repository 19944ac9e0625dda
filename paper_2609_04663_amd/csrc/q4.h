// Products of a few rows with matrices in 4 bits, Y[r] = X[r] W[e(r)]^T, and the
// packing of those matrices.
//
// Arithmetic.  An integer q of a weight becomes the exact 16 + q in the matrix
// instruction's type with one shift and one and-or for two weights (its four
// bits below the exponent of 16), so a group's sum is sum (16 + q) x in FP32,
// and s (q - 8) summed over a group is s times that sum started at -24 sum x
// (-16 sum x with offsets, plus m sum x).  The sums of x per group are made once
// where x is staged.  FP32 rows are three BF16 components (Eq. fp32split) and
// three products with the same weights.  No weight is rounded.
//
// Shape.  v_mfma 16 x 16 x 32 with tokens as rows and weight rows as columns: a
// lane loads 16 bytes, 32 indices of one weight row; four lanes of a row hold
// 128, and a 4 x 4 exchange between them (two v_permlane32_swap, two
// v_permlane16_swap) makes each instruction span one run of 32, so that groups
// of 32 can be scaled.  The waves of a workgroup share the reduction (and
// the columns, where x leaves room in LDS for few indices only) and add up
// their sums in LDS at the end.
#pragma once

#include "api_state.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <typename T>
using frag = T __attribute__((ext_vector_type(8)));

constexpr int WAVES = 8, BLOCK = 128;       // waves of a workgroup; indices of a lane quad

template <typename T>
struct Q4Elem {
    using comp = T;
    static constexpr int PLANES = 1;
};
template <>
struct Q4Elem<float> {
    using comp = bhalf;
    static constexpr int PLANES = 3;
};

__device__ __forceinline__ f32x4 mfma16(frag<bhalf> a, frag<bhalf> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(frag<half> a, frag<half> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// 16 + q of the eight 4-bit fields of w, fields (0, 4), (1, 5), (2, 6), (3, 7)
// in the pairs of the result.  16 is 0x4180 in bfloat16 (field at bit 3) and
// 0x4C00 in half (field at bit 6).
template <typename C>
__device__ __forceinline__ frag<C> sixteen_plus(unsigned w) {
    constexpr bool BF = std::is_same<C, bhalf>::value;
    constexpr unsigned MASK = BF ? 0x00780078u : 0x03C003C0u, ONE = BF ? 0x41804180u : 0x4C004C00u;
    constexpr int UP = BF ? 3 : 6;
    u32x4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const unsigned v = 4 * p < UP ? w << (UP - 4 * p) : w >> (4 * p - UP);
        r[p] = (v & MASK) | ONE;
    }
    return __builtin_bit_cast(frag<C>, r);
}
// where element i of eight consecutive ones goes to match it
__device__ __forceinline__ constexpr int field_place(int i) { return i % 4 * 2 + i / 4; }

// Lane quarter h of register i gets quarter i's register h.
__device__ __forceinline__ void exchange_quarters(unsigned (&d)[4]) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32x2 r = __builtin_amdgcn_permlane32_swap(d[i], d[i + 2], false, false);
        d[i] = r[0];
        d[i + 2] = r[1];
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const u32x2 r = __builtin_amdgcn_permlane16_swap(d[i], d[i + 1], false, false);
        d[i] = r[0];
        d[i + 1] = r[1];
    }
}

// What a launch fixes for all of its workgroups.
struct Q4Plan {
    int wk;                         // waves along the reduction, of 8; the others are along the columns
    int chunk;                      // blocks of 128 indices that x is staged for at a time
    int tokens;                     // most rows of a tile
    int splits;                     // workgroups along the reduction
    float *part;                    // splits x R x N sums where splits > 1
};

template <typename T>
constexpr int lds_bytes() { return Q4Elem<T>::PLANES == 3 ? 128 * 1024 : 64 * 1024; }

// A tile of MT x 16 rows, NT tiles of 16 columns of a wave, groups of G.  FEW: the
// tile has at most four rows (MT = 1): row t of the instruction is token t / 4,
// so that the tokens of a lane's quarter are in one accumulator register instead of
// four, and the work per group is a quarter.
template <typename T, int MT, int NT, int G, bool FEW>
__device__ __forceinline__ void q4_tile(const Q4Gemm &g, const Q4Plan &p, const RowTile &t, char *lds) {
    using C = typename Q4Elem<T>::comp;
    constexpr int PL = Q4Elem<T>::PLANES, U = 4 / NT, GB = BLOCK / G;    // blocks of a set; groups of a block
    constexpr int REGS = FEW ? 1 : 4, TOKENS = FEW ? 4 : 16 * MT;
    typedef float sums_t __attribute__((ext_vector_type(REGS)));         // of a lane's tokens
    const int wk = p.wk, wn = WAVES / wk, cols = 16 * NT * wn;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int my_n = wave % wn, my_k = wave / wn, h = lane >> 4;
    const int m = (int)(t.end - t.first), K = g.K, N = g.N, col0 = t.col * cols;
    float *const part = p.part ? p.part + (int64_t)blockIdx.y * g.R * N : nullptr;
    T *const Y = static_cast<T *>(g.Y);
    auto put = [&](int tok, int col, float v) {
        if (part) part[(t.first + tok) * N + col] = v;
        else Y[(t.first + tok) * g.ldy + col] = (T)v;
    };
    if (t.e == g.E) {                                 // rows of no expert
        for (int i = threadIdx.x; i < m * cols; i += 64 * WAVES)
            if (col0 + i % cols < N) put(i / cols, col0 + i % cols, 0.0f);
        return;
    }
    const int groups = K / G, blocks = (K + BLOCK - 1) / BLOCK;
    const int per = (blocks + p.splits - 1) / p.splits;
    const int b_lo = blockIdx.y * per, b_hi = b_lo + per < blocks ? b_lo + per : blocks;
    const uint8_t *q_row[NT];
    const T *s_row[NT], *m_row[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int n = col0 + (my_n * NT + i) * 16 + (lane & 15);
        const int64_t at = (int64_t)t.e * N + (n < N ? n : N - 1);
        q_row[i] = g.Q + at * (K / 2) + 16 * h;
        s_row[i] = static_cast<const T *>(g.scales) + at * groups;
        m_row[i] = g.mins ? static_cast<const T *>(g.mins) + at * groups : nullptr;
    }
    // a set: U neighbouring blocks of the wave's NT column tiles.  The scales of
    // all of them are one load: 16 rows of a few bytes cost the address unit as
    // much as 16 rows of 64.
    struct Set {
        vec<unsigned, 4> w[U][NT];
        vec<T, U * GB> s[NT], o[NT];
    };
    auto load_groups = [&](const T *row, int b) {
        vec<T, U * GB> v;
        if (b * GB + U * GB <= groups) {
            v = *reinterpret_cast<const vec<T, U * GB> *>(row + b * GB);
        } else {
#pragma unroll
            for (int i = 0; i < U * GB; ++i) v[i] = row[b * GB + i < groups ? b * GB + i : groups - 1];
        }
        return v;
    };
    auto block_of = [&](int set, int u) { return b_lo + (set * wk + my_k) * U + u; };
    auto load = [&](Set &x, int set) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int want = block_of(set, u), b = want < b_hi ? want : b_hi - 1;
            // a run of 32 past the end is read from the row's start and not used
            const int at = b * BLOCK + 32 * h < K ? b * (BLOCK / 2) : -16 * h;
#pragma unroll
            for (int i = 0; i < NT; ++i)
                x.w[u][i] = __builtin_nontemporal_load(reinterpret_cast<const vec<unsigned, 4> *>(q_row[i] + at));
        }
        const int b = block_of(set, 0);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            x.s[i] = load_groups(s_row[i], b);
            if (g.mins) x.o[i] = load_groups(m_row[i], b);
        }
    };
    const float start = g.mins ? -16.0f : -24.0f;
    const int RS = p.chunk * BLOCK * 2 + 16;
    float *const sums = reinterpret_cast<float *>(lds + PL * p.tokens * RS);
    const int in_chunk = p.chunk / (wk * U);                        // sets
    const int sets = b_hi > b_lo ? (b_hi - b_lo + wk * U - 1) / (wk * U) : 0;
    sums_t y[NT][MT] = {};
    int tok_at[MT];
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int tok = FEW ? (lane & 15) / 4 : 16 * a + (lane & 15);
        tok_at[a] = (tok < m ? tok : m - 1) * RS + h * 16;
    }
    Set now, next;
    if (sets > 0) load(now, 0);
    for (int set = 0; set < sets; ++set) {
        if (set % in_chunk == 0) {
            const int c0 = (b_lo + set * U * wk) * BLOCK;
            const int len = K - c0 < p.chunk * BLOCK ? K - c0 : p.chunk * BLOCK;
            const int runs = len / 8;
            if (set > 0) __syncthreads();
            // stage x: a thread takes eight indices of a token
            for (int u = threadIdx.x; u < m * runs; u += 64 * WAVES) {
                const int tok = u / runs, k = u % runs * 8;
                const int64_t r = t.first + tok, at = g.rows ? g.rows[r] : r;
                frag<float> x = frag<float>{};
                if (at >= 0 && at < g.xrows) {
                    const vec<T, 8> v = *reinterpret_cast<const vec<T, 8> *>(
                        static_cast<const T *>(g.X) + at * g.ldx + c0 + k);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
                }
                float sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                // the threads of a group are neighbours, and all of them are here: len is whole groups
#pragma unroll
                for (int d = 1; d < G / 8; d <<= 1) sum += __shfl_xor(sum, d);
                if (k % G == 0) sums[k / G * TOKENS + tok] = sum * start;
                frag<float> v;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[field_place(i)] = x[i];
#pragma unroll
                for (int c = 0; c < PL; ++c) {
                    const frag<C> f = __builtin_convertvector(v, frag<C>);
                    *reinterpret_cast<frag<C> *>(lds + (c * p.tokens + tok) * RS + k * 2) = f;
                    if (c + 1 < PL) v = v - __builtin_convertvector(f, frag<float>);
                }
            }
            __syncthreads();
        }
        if (set + 1 < sets) load(next, set + 1);
        // block u of the set; whole: all of its indices are there
        auto multiply = [&](int u, auto whole) __attribute__((always_inline)) {
            const int b = block_of(set, u);
            const int in = (set % in_chunk * wk + my_k) * U + u;       // block of the chunk
            unsigned w[NT][4];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) w[i][j] = now.w[u][i][j];
                exchange_quarters(w[i]);
            }
            f32x4 acc[NT][MT];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!decltype(whole)::value && b * BLOCK + 32 * j >= K) break;
                const float *const sum = sums + (in * GB + 32 * j / G) * TOKENS + REGS * h;
                if (32 * j % G == 0) {
#pragma unroll
                    for (int a = 0; a < MT; ++a) {
                        const sums_t v = *reinterpret_cast<const sums_t *>(sum + 16 * a);
                        f32x4 c = {};
#pragma unroll
                        for (int r = 0; r < REGS; ++r) c[r] = v[r];
#pragma unroll
                        for (int i = 0; i < NT; ++i) acc[i][a] = c;
                    }
                }
                frag<C> x[MT][PL];
#pragma unroll
                for (int a = 0; a < MT; ++a)
#pragma unroll
                    for (int c = 0; c < PL; ++c)
                        x[a][c] = *reinterpret_cast<const frag<C> *>(lds + tok_at[a] + c * p.tokens * RS +
                                                                     (in * BLOCK + 32 * j) * 2);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const frag<C> wf = sixteen_plus<C>(w[i][j]);
#pragma unroll
                    for (int c = PL - 1; c >= 0; --c)
#pragma unroll
                        for (int a = 0; a < MT; ++a) acc[i][a] = mfma16(x[a][c], wf, acc[i][a]);
                }
                if ((32 * j + 32) % G == 0) {
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const float s = (float)now.s[i][u * GB + 32 * j / G];
#pragma unroll
                        for (int a = 0; a < MT; ++a)
#pragma unroll
                            for (int r = 0; r < REGS; ++r) y[i][a][r] = fmaf(acc[i][a][r], s, y[i][a][r]);
                        if (g.mins) {
                            const float o = (float)now.o[i][u * GB + 32 * j / G] * (1.0f / -16.0f);    // of start
#pragma unroll
                            for (int a = 0; a < MT; ++a) {
                                const sums_t v = *reinterpret_cast<const sums_t *>(sum + 16 * a);
#pragma unroll
                                for (int r = 0; r < REGS; ++r) y[i][a][r] = fmaf(v[r], o, y[i][a][r]);
                            }
                        }
                    }
                }
            }
        };
        if (block_of(set, U - 1) < b_hi && (block_of(set, U - 1) + 1) * BLOCK <= K) {
#pragma unroll
            for (int u = 0; u < U; ++u) multiply(u, std::true_type{});
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (block_of(set, u) < b_hi) multiply(u, std::false_type{});
        }
        now = next;
    }
    // the sums of the waves along the reduction, in order
    float *const share = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        __syncthreads();
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int r = 0; r < REGS; ++r)
                share[(wave * MT + a) * 256 + (REGS * h + r) * 16 + (lane & 15)] = y[i][a][r];
        __syncthreads();
        for (int j = threadIdx.x; j < m * 16 * wn; j += 64 * WAVES) {
            const int tok = j / (16 * wn), n = j / 16 % wn, c = j % 16, col = col0 + (n * NT + i) * 16 + c;
            if (col >= N) continue;
            float v = 0.0f;
            for (int w = 0; w < wk; ++w)
                v += share[((w * wn + n) * MT + tok / 16) * 256 + tok % 16 * 16 + c];
            put(tok, col, v);
        }
    }
}

template <typename T, int MT, int NT, int G>
__global__ __launch_bounds__(64 * WAVES) void q4_gemm_kernel(Q4Gemm g, Q4Plan p) {
    __shared__ __attribute__((aligned(16))) char lds[lds_bytes<T>()];
    const int cols = 16 * NT * (WAVES / p.wk);
    const RowTile t = RowTiles(g.offsets, g.E, g.R, 16 * MT, (g.N + cols - 1) / cols).at(blockIdx.x);
    if (t.e < 0) return;
    if (MT == 1 && t.end - t.first <= 4) q4_tile<T, MT, NT, G, MT == 1>(g, p, t, lds);
    else q4_tile<T, MT, NT, G, false>(g, p, t, lds);
}

// Y = the sum of the parts, in order.
template <typename T>
__global__ __launch_bounds__(256) void q4_join_kernel(const float *__restrict__ part, int splits, int64_t R,
                                                      int N, T *__restrict__ Y, int64_t ldy) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = R * N;
    if (i >= n) return;
    float v = part[i];
    for (int s = 1; s < splits; ++s) v += part[s * n + i];
    Y[i / N * ldy + i % N] = (T)v;
}

}  // namespace

namespace {

// Row tiles that an even load of the rows would give, for choices that need not
// be exact.
int64_t likely_tiles(const Q4Gemm &g, int rows) {
    const int64_t reached = g.E < g.R ? g.E : g.R, full = g.R / rows;
    return full > reached ? full : reached;
}

template <typename T, int MT, int NT>
Q4Plan plan_q4(const Q4Gemm &g) {
    constexpr int U = 4 / NT;
    Q4Plan p = {};
    p.tokens = g.R < 16 * MT ? (int)g.R : 16 * MT;
    const int blocks = (g.K + BLOCK - 1) / BLOCK;
    const int each = Q4Elem<T>::PLANES * p.tokens * 2 * BLOCK + 16 * MT * 4 * (BLOCK / g.group);
    const int fit = (lds_bytes<T>() - 16 * Q4Elem<T>::PLANES * p.tokens) / each;
    // waves along the columns, as long as there are WAVES_MIN waves for the chip
    constexpr int64_t WAVES_MIN = 16 * 256;
    p.wk = WAVES;
    while (p.wk > 1 && (p.wk * U > fit ||
                        likely_tiles(g, 16 * MT) * ((g.N + 16 * NT * 2 * (WAVES / p.wk) - 1) /
                                                    (16 * NT * 2 * (WAVES / p.wk))) * WAVES >= WAVES_MIN))
        p.wk /= 2;
    const int step = p.wk * U, need = (blocks + step - 1) / step * step;
    p.chunk = fit / step * step;
    if (p.chunk > need) p.chunk = need;
    if (p.chunk < step) p.chunk = step;               // K = 0
    // few workgroups with long reductions: more along the reduction
    const int cols = 16 * NT * (WAVES / p.wk);
    const int64_t tiles = likely_tiles(g, 16 * MT) * ((g.N + cols - 1) / cols);
    p.splits = 1;
    while (p.splits < 16 && tiles * p.splits * 2 <= 256 && blocks / (p.splits * 2) >= 4 * step) p.splits *= 2;
    return p;
}

}  // namespace

template <typename T>
hipError_t run_q4_gemm(const Q4Gemm &g, hipStream_t s) {
    hipError_t e = hipSuccess;
    auto run = [&](auto mt, auto nt, auto group) {
        constexpr int MT = decltype(mt)::value, NT = decltype(nt)::value;
        Q4Plan p = plan_q4<T, MT, NT>(g);
        if (p.splits > 1) {
            char *w = nullptr;
            if (api_workspace(sizeof(float) * p.splits * g.R * g.N, &w) != EMU_OK) {
                api_clear_error();
                p.splits = 1;       // no memory: one workgroup for the whole reduction
            }
            p.part = reinterpret_cast<float *>(w);
        }
        const int cols = 16 * NT * (WAVES / p.wk);
        const int64_t tiles = row_blocks_bound(g.R, g.E, 16 * MT) * ((g.N + cols - 1) / cols);
        q4_gemm_kernel<T, MT, NT, decltype(group)::value><<<dim3((unsigned)tiles, p.splits), 64 * WAVES, 0, s>>>(g, p);
        e = hipGetLastError();
        if (e == hipSuccess && p.splits > 1) {
            q4_join_kernel<T><<<(unsigned)((g.R * g.N + 255) / 256), 256, 0, s>>>(p.part, p.splits, g.R, g.N,
                                                                                  static_cast<T *>(g.Y), g.ldy);
            e = hipGetLastError();
        }
    };
    auto rows = [&](auto group) {
        using std::integral_constant;
        const integral_constant<int, 1> one;
        const integral_constant<int, 2> two;
        const integral_constant<int, 3> three;
        const integral_constant<int, 4> four;
        if (g.R <= 16 * (int64_t)g.E) run(one, one, group);
        else if (g.R <= 32 * (int64_t)g.E) run(two, four, group);
        else if (g.R <= 48 * (int64_t)g.E) run(three, integral_constant<int, Q4Elem<T>::PLANES == 3 ? 2 : 4>{}, group);
        else run(four, two, group);
    };
    if (g.group == 32) rows(std::integral_constant<int, 32>{});
    else if (g.group == 64) rows(std::integral_constant<int, 64>{});
    else rows(std::integral_constant<int, 128>{});
    return e;
}

}  // namespace emu
