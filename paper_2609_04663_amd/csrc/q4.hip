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

// LDS of a workgroup: PLANES x tokens x (chunk + 8) components, then per group
// of the chunk 16 MT sums of x.
template <typename T>
__host__ __device__ inline int q4_x_bytes(int tokens, int chunk) {
    return Q4Elem<T>::PLANES * tokens * (chunk * 2 + 16);
}

template <typename T, int MT>
__global__ __launch_bounds__(64 * WAVES) void q4_gemm_kernel(
    const T *__restrict__ X, int64_t ldx, int64_t xrows, const int *__restrict__ rows,
    const uint8_t *__restrict__ Q, const T *__restrict__ scales, const T *__restrict__ mins,
    const int *__restrict__ offsets, int E, int64_t R, T *__restrict__ Y, int64_t ldy, int N, int K,
    int group, int chunk, int tokens_max, int wk) {
    using C = typename Q4Elem<T>::comp;
    constexpr int PL = Q4Elem<T>::PLANES;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int wn = WAVES / wk, cols = 16 * wn;
    const RowTile t = RowTiles(offsets, E, R, 16 * MT, (N + cols - 1) / cols).at(blockIdx.x);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int my_n = wave % wn, my_k = wave / wn, h = lane >> 4;
    const int m = (int)(t.end - t.first);
    const int n = t.col * cols + my_n * 16 + (lane & 15), nc = n < N ? n : N - 1;
    if (t.e == E) {                                   // rows of no expert
        for (int i = threadIdx.x; i < m * cols; i += 64 * WAVES) {
            const int c = t.col * cols + i % cols;
            if (c < N) Y[(t.first + i / cols) * ldy + c] = T(0.0f);
        }
        return;
    }
    const int groups = K / group;
    const uint8_t *const q_row = Q + ((int64_t)t.e * N + nc) * (K / 2) + 16 * h;
    const T *const s_row = scales + ((int64_t)t.e * N + nc) * groups;
    const T *const m_row = mins ? mins + ((int64_t)t.e * N + nc) * groups : nullptr;
    const float start = mins ? -16.0f : -24.0f;
    const int RS = chunk * 2 + 16;
    float *const sums = reinterpret_cast<float *>(lds + q4_x_bytes<T>(tokens_max, chunk));
    f32x4 y[MT] = {};
    for (int c0 = 0; c0 < K; c0 += chunk) {
        const int len = K - c0 < chunk ? K - c0 : chunk;
        __syncthreads();
        // stage x: a thread takes eight indices of a token
        for (int u = threadIdx.x; u < m * (len / 8); u += 64 * WAVES) {
            const int tok = u / (len / 8), k = u % (len / 8) * 8;
            const int64_t r = t.first + tok, at = rows ? rows[r] : r;
            frag<float> x = frag<float>{};
            if (at >= 0 && at < xrows) {
                const vec<T, 8> v = *reinterpret_cast<const vec<T, 8> *>(X + at * ldx + c0 + k);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
            }
            float sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            // the threads of a group are neighbours, and all of them are here: len is whole groups
            for (int d = 1; d < group / 8; d <<= 1) sum += __shfl_xor(sum, d);
            if (k % group == 0) sums[k / group * (16 * MT) + tok] = sum;
            frag<float> p;
#pragma unroll
            for (int i = 0; i < 8; ++i) p[field_place(i)] = x[i];
#pragma unroll
            for (int c = 0; c < PL; ++c) {
                const frag<C> v = __builtin_convertvector(p, frag<C>);
                *reinterpret_cast<frag<C> *>(lds + (c * tokens_max + tok) * RS + k * 2) = v;
                if (c + 1 < PL) p = p - __builtin_convertvector(v, frag<float>);
            }
        }
        __syncthreads();
        for (int b = my_k * BLOCK; b < len; b += wk * BLOCK) {
            unsigned w[4] = {};
            if (b + 32 * h < len) {
                const vec<unsigned, 4> v =
                    *reinterpret_cast<const vec<unsigned, 4> *>(q_row + (c0 + b) / 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = v[i];
            }
            exchange_quarters(w);
            f32x4 acc[MT];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = b + 32 * i;
                if (k >= len) break;
                if (k % group == 0) {
#pragma unroll
                    for (int a = 0; a < MT; ++a)
                        acc[a] = *reinterpret_cast<const f32x4 *>(sums + k / group * (16 * MT) + 16 * a + 4 * h) * start;
                }
                const frag<C> wf = sixteen_plus<C>(w[i]);
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    const int tok = 16 * a + (lane & 15);
                    const char *const xp = lds + (tok < m ? tok : m - 1) * RS + (k + 8 * h) * 2;
#pragma unroll
                    for (int c = PL - 1; c >= 0; --c)
                        acc[a] = mfma16(*reinterpret_cast<const frag<C> *>(xp + c * tokens_max * RS), wf, acc[a]);
                }
                if ((k + 32) % group == 0) {
                    const int g = (c0 + k) / group;
                    const float s = (float)s_row[g];
#pragma unroll
                    for (int a = 0; a < MT; ++a) y[a] += acc[a] * s;
                    if (m_row) {
                        const float o = (float)m_row[g];
#pragma unroll
                        for (int a = 0; a < MT; ++a)
                            y[a] += *reinterpret_cast<const f32x4 *>(sums + k / group * (16 * MT) + 16 * a + 4 * h) * o;
                    }
                }
            }
        }
    }
    // the sums of the waves along the reduction, in order
    __syncthreads();
    float *const part = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            part[(wave * MT + a) * 256 + (4 * h + r) * 16 + (lane & 15)] = y[a][r];
    __syncthreads();
    for (int i = threadIdx.x; i < m * cols; i += 64 * WAVES) {
        const int tok = i / cols, c = i % cols, col = t.col * cols + c;
        if (col >= N) continue;
        float v = 0.0f;
        for (int w = 0; w < wk; ++w)
            v += part[((w * wn + c / 16) * MT + tok / 16) * 256 + tok % 16 * 16 + c % 16];
        Y[(t.first + tok) * ldy + col] = (T)v;
    }
}

// A thread packs eight entries; the threads of a group are neighbours.
template <typename T>
__global__ __launch_bounds__(256) void q4_pack_kernel(const T *__restrict__ W, int64_t rows, int64_t ldw,
                                                      int K, int group, uint8_t *__restrict__ Q,
                                                      T *__restrict__ scales) {
    const int64_t per = K / 8, u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= rows * per) return;
    const int64_t r = u / per, k = u % per * 8;
    float x[8], top = 0.0f;
    load_f32<8>(W + r * ldw + k, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
    for (int d = 1; d < group / 8; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const T stored = (T)(top / 7.0f);
    const float s = (float)stored;
    unsigned q = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = s > 0.0f ? fminf(fmaxf(rintf(x[i] / s), -8.0f), 7.0f) : 0.0f;
        q |= (unsigned)((int)v + 8) << (4 * i);
    }
    *reinterpret_cast<vec<uint8_t, 4> *>(Q + r * (K / 2) + k / 2) = __builtin_bit_cast(vec<uint8_t, 4>, q);
    if (k % group == 0) scales[r * (K / group) + k / group] = stored;
}

}  // namespace

hipError_t launch_q4_gemm(const Q4Gemm &g, hipStream_t s) {
    with_type(g.dtype, [&](auto z) {
        using T = decltype(z);
        auto run = [&](auto mt) {
            constexpr int MT = decltype(mt)::value;
            const int tokens = g.R < 16 * MT ? (int)g.R : 16 * MT;
            // as many indices of x at a time as 56 KB hold
            const int per = Q4Elem<T>::PLANES * tokens * 2 * BLOCK + 16 * MT * 4 * (BLOCK / g.group);
            int blocks = (56 * 1024 - 16 * Q4Elem<T>::PLANES * tokens) / per;
            const int all = (g.K + BLOCK - 1) / BLOCK;
            if (blocks > all) blocks = all;
            int wk = WAVES;
            while (wk > 1 && wk > blocks) wk /= 2;
            if (blocks > wk) blocks = blocks / wk * wk;
            const int chunk = blocks * BLOCK;
            const int cols = 16 * (WAVES / wk);
            int bytes = q4_x_bytes<T>(tokens, chunk) + chunk / g.group * 16 * MT * 4;
            if (bytes < WAVES * MT * 1024) bytes = WAVES * MT * 1024;
            const int64_t tiles = row_blocks_bound(g.R, g.E, 16 * MT) * ((g.N + cols - 1) / cols);
            q4_gemm_kernel<T, MT><<<(unsigned)tiles, 64 * WAVES, bytes, s>>>(
                static_cast<const T *>(g.X), g.ldx, g.xrows, g.rows, g.Q,
                static_cast<const T *>(g.scales), static_cast<const T *>(g.mins), g.offsets, g.E, g.R,
                static_cast<T *>(g.Y), g.ldy, g.N, g.K, g.group, chunk, tokens, wk);
        };
        if (g.R <= 16 * (int64_t)g.E) run(std::integral_constant<int, 1>{});
        else run(std::integral_constant<int, 3>{});
    });
    return hipGetLastError();
}

hipError_t launch_q4_pack(int dtype, const void *W, int64_t rows, int64_t ldw, int K, int group,
                          uint8_t *Q, void *scales, hipStream_t s) {
    with_type(dtype, [&](auto z) {
        using T = decltype(z);
        q4_pack_kernel<T><<<(unsigned)((rows * (K / 8) + 255) / 256), 256, 0, s>>>(
            static_cast<const T *>(W), rows, ldw, K, group, Q, static_cast<T *>(scales));
    });
    return hipGetLastError();
}

}  // namespace emu
