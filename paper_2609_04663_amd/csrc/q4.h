// Products of a few rows with matrices in 4 bits, Y[r] = X[r] W[e(r)]^T.
//
// Arithmetic.  An integer q of a weight becomes the exact 16 + q in the matrix
// instruction's type with a shift, an and, and an or for two weights (its four
// bits below the exponent of 16), so a group's sum is sum (16 + q) x in FP32, and
// s (q - 8) summed over the group is s times (that sum - 24 sum x); with offsets
// s times (that sum - 16 sum x) plus m sum x.  FP32 rows are three BF16 components
// (Eq. fp32split) and three products with the same weights.  No weight is rounded.
//
// Shape.  v_mfma 16 x 16 x 32 with tokens as rows and weight rows as columns: a
// lane loads 16 bytes, 32 indices of one weight row; four lanes of a row hold
// 128, and a 4 x 4 exchange between them (two v_permlane32_swap, two
// v_permlane16_swap) makes each instruction span one run of 32, so that groups
// of 32 can be scaled.  x lies in LDS, the 16-byte units of token t permuted by
// t % 16, so that the 16 tokens of a read touch every bank once.  Two forms:
//   prepared (FP32, and tiles of at most four rows): the components in the order
//     of the weights' fields, with the sums of each group, made as x is staged; of
//     more than 16 FP32 rows a chunk ahead, loaded to registers under the products
//     of the chunk before.  What that costs is the same for every workgroup, so all
//     eight waves lie along the columns there: 40 rows of 8192 x 8192 42 us, with
//     two waves along the reduction and no fetching ahead 50;
//   raw (more rows of 16 bits): copied as it is by global_load_lds, a chunk ahead
//     in a second buffer where it does not fit at once; a fragment is put into the
//     fields' order after it is read, and one more matrix instruction with ones
//     gives the sums.  16 rows of 16384 x 16384: 63 us, prepared 84; one row of
//     64 matrices of 4096 x 4096: 136 us, prepared 116.
// The waves of a workgroup share the reduction (and the columns, where x leaves
// room for few indices only) and add up their sums in LDS at the end.
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
// 0x4C00 in half (field at bit 6).  The mask comes in a register, so that a shift and one
// v_and_or_b32 make a pair (two constants would be two instructions).
template <typename C>
__device__ __forceinline__ unsigned field_mask() {
    unsigned m = std::is_same<C, bhalf>::value ? 0x00780078u : 0x03C003C0u;
    asm("" : "+v"(m));
    return m;
}
template <typename C>
__device__ __forceinline__ frag<C> sixteen_plus(unsigned w, unsigned mask) {
    constexpr bool BF = std::is_same<C, bhalf>::value;
    constexpr unsigned ONE = BF ? 0x41804180u : 0x4C004C00u;
    constexpr int UP = BF ? 3 : 6;
    u32x4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const unsigned v = 4 * p < UP ? w << (UP - 4 * p) : w >> (4 * p - UP);
        r[p] = (v & mask) | ONE;
    }
    return __builtin_bit_cast(frag<C>, r);
}
// Eight consecutive entries of x in the order that matches it.
template <typename C>
__device__ __forceinline__ frag<C> to_fields(frag<C> x) {
    const u32x4 r = __builtin_bit_cast(u32x4, x);
    u32x4 f;
    f[0] = __builtin_amdgcn_perm(r[2], r[0], 0x05040100u);      // entries 0, 4
    f[1] = __builtin_amdgcn_perm(r[2], r[0], 0x07060302u);      // 1, 5
    f[2] = __builtin_amdgcn_perm(r[3], r[1], 0x05040100u);      // 2, 6
    f[3] = __builtin_amdgcn_perm(r[3], r[1], 0x07060302u);      // 3, 7
    return __builtin_bit_cast(frag<C>, f);
}

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
    int passes;                     // column tiles of a workgroup, one after the other
    int splits;                     // workgroups along the reduction
    float *part;                    // splits x R x N sums where splits > 1
    bool copies;                    // X is 16-byte aligned
};

// LDS: x, one buffer or two (prepared: with its sums per group); and 1 KB for
// each wave and tile of 16 rows, where the waves along the reduction add up.
template <typename T, int MT>
constexpr int lds_bytes() { return (Q4Elem<T>::PLANES == 3 ? 152 : (MT == 1 ? 72 : 128)) * 1024; }
template <typename T, int MT>
constexpr int share_at() { return lds_bytes<T, MT>() - WAVES * MT * 1024; }
// bytes of a buffer for `chunk` blocks of 128 indices of m tokens: components (the
// copies write whole KB), and sums for `slots` tokens
template <typename T>
__host__ __device__ constexpr int sums_at(int m, int chunk) {
    return (Q4Elem<T>::PLANES * m * chunk * 256 + 1023) / 1024 * 1024;
}
template <typename T>
__host__ __device__ constexpr int buffer_bytes(int m, int slots, int group, int chunk) {
    return sums_at<T>(m, chunk) + chunk * (BLOCK / group) * slots * 4;
}
// blocks that a buffer of the given size holds
template <typename T>
__host__ __device__ constexpr int blocks_that_fit(int m, int slots, int group, int bytes) {
    return (bytes - 1024) / (Q4Elem<T>::PLANES * m * 256 + BLOCK / group * slots * 4);
}

// Sixteen zero bytes: rows outside.
__device__ __attribute__((aligned(16))) float g_zero16[4];

// A tile of MT x 16 rows, NT tiles of 16 columns of a wave, sets of U blocks of
// 128 indices, groups of G.  FEW: the tile has at most four rows (MT = 1): row t
// of the instruction is token t / 4, so that the tokens of a lane's quarter are in
// one accumulator register instead of four, and the work per group is a quarter.
template <typename T, int MT, int NT, int U, int G, bool FEW>
__device__ __forceinline__ void q4_tile(const Q4Gemm &g, const Q4Plan &p, const RowTile &t, char *lds) {
    using C = typename Q4Elem<T>::comp;
    constexpr int PL = Q4Elem<T>::PLANES, GB = BLOCK / G;                // groups of a block
    constexpr int REGS = FEW ? 1 : 4, TOKENS = FEW ? 4 : 16 * MT;
    constexpr bool RAW = PL == 1 && !FEW;
    constexpr bool FETCH = PL == 3 && MT > 1;         // prepared a chunk ahead, through registers
    constexpr int SLOTS = RAW ? 0 : TOKENS;                              // sums of a group
    constexpr int THREADS = 64 * WAVES;
    static_assert(blocks_that_fit<T>(16 * MT, 16 * MT, 32, share_at<T, MT>()) >= U, "a set's blocks");
    typedef float sums_t __attribute__((ext_vector_type(REGS)));         // of a lane's tokens
    const int wk = p.wk, wn = WAVES / wk, cols = 16 * NT * wn;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int my_n = wave % wn, my_k = wave / wn, h = lane >> 4;
    const int m = (int)(t.end - t.first), K = g.K, N = g.N;
    const int col0 = t.col * cols * p.passes;
    float *const part = p.part ? p.part + (int64_t)blockIdx.y * g.R * N : nullptr;
    T *const Y = static_cast<T *>(g.Y);
    float odd = 0.0f;                                 // NaN where a result was not finite
    auto put = [&](int tok, int col, float v) {
        odd = fmaf(v, 0.0f, odd);
        if (part) part[(t.first + tok) * N + col] = v;
        else Y[(t.first + tok) * g.ldy + col] = (T)v;
    };
    const int left = (N - col0 + cols - 1) / cols, passes = left < p.passes ? left : p.passes;
    if (t.e == g.E) {                                 // rows of no expert
        for (int i = threadIdx.x; i < m * cols * passes; i += THREADS) {
            const int c = col0 + i % (cols * passes);
            if (c < N) put(i / (cols * passes), c, 0.0f);
        }
        return;
    }
    const int groups = K / G, blocks = (K + BLOCK - 1) / BLOCK;
    const int per = (blocks + p.splits - 1) / p.splits;
    const int b_lo = blockIdx.y * per, b_hi = b_lo + per < blocks ? b_lo + per : blocks;
    const int step = wk * U, sets = b_hi > b_lo ? (b_hi - b_lo + step - 1) / step : 0;

    // x: all of it at once, staged for every pass; or a chunk at a time, in two
    // buffers where it is copied or fetched ahead
    const int mine = b_hi > b_lo ? b_hi - b_lo : 0;
    const bool once = buffer_bytes<T>(m, SLOTS, G, mine) <= share_at<T, MT>();
    const bool copies = RAW && p.copies;
    const int two = blocks_that_fit<T>(m, SLOTS, G, share_at<T, MT>() / 2) / step * step;
    const bool ahead = !once && (copies || FETCH) && two > 0;
    const int chunk = once ? mine : (ahead ? two : blocks_that_fit<T>(m, SLOTS, G, share_at<T, MT>()) / step * step);
    const int in_chunk = once ? (sets > 0 ? sets : 1) : chunk / step;    // sets
    const int RB = chunk * 256, sums_in = sums_at<T>(m, chunk);          // bytes of a token's components
    const int buf_bytes = sums_in + chunk * GB * SLOTS * 4;
    const float start = g.mins ? -16.0f : -24.0f;
    const int k_hi = b_hi * BLOCK < K ? b_hi * BLOCK : K;
    // the row of each token, looked up once
    __shared__ int row_of[16 * MT];
    if ((int)threadIdx.x < m) {
        const int64_t r = t.first + threadIdx.x, at = g.rows ? g.rows[r] : r;
        row_of[threadIdx.x] = at >= 0 && at < g.xrows ? (int)at : -1;
    }
    // unit u (eight entries) of a token lies at (u ^ token % 16)
    auto place = [&](int c, int tok, int unit) { return (c * m + tok) * RB + ((unit ^ (tok & 15)) << 4); };
    // starts the copies of the chunk from block b on
    auto copy = [&](char *buf, int b) {
        const int units = chunk * 16, total = m * units;
        for (int c = wave; c * 64 < total; c += WAVES) {
            const int i = c * 64 + lane < total ? c * 64 + lane : total - 1, tok = i / units;
            const int k = b * BLOCK + ((i - tok * units) ^ (tok & 15)) * 8;
            const int kc = k < k_hi ? k : b * BLOCK;  // past the end: something, not used
            const T *const src = row_of[tok] < 0 ? reinterpret_cast<const T *>(g_zero16)
                                                 : static_cast<const T *>(g.X) + row_of[tok] * g.ldx + kc;
            copy_lanes(reinterpret_cast<const char *>(src), buf + c * 1024);
        }
    };
    // the same by loads and stores, prepared on the way; the threads of a group
    // are neighbours, and all of them are here: a chunk is whole groups
    // Puts entries v of a token, unit u of the chunk, into the buffer.
    auto prepare = [&](char *buf, int tok, int unit, const vec<T, 8> &v) {
        if constexpr (RAW) {
            *reinterpret_cast<vec<T, 8> *>(buf + place(0, tok, unit)) = v;
        } else {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
            float sum = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
            sum += moved<0xB1>(sum);                  // over the group's lanes
            sum += moved<0x4E>(sum);
            if constexpr (G >= 64) sum += moved<0x141>(sum);
            if constexpr (G >= 128) sum += moved<0x140>(sum);
            if (unit % (G / 8) == 0)
                reinterpret_cast<float *>(buf + sums_in)[unit / (G / 8) * TOKENS + tok] = sum * start;
#pragma unroll
            for (int c = 0; c < PL; ++c) {
                u32x4 w;                              // in the fields' order
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    typedef C c2 __attribute__((ext_vector_type(2)));
                    const c2 pair = {(C)f[i], (C)f[i + 4]};
                    w[i] = __builtin_bit_cast(unsigned, pair);
                    if (c + 1 < PL) {                 // (three components: of bfloat16)
                        f[i] -= __uint_as_float(w[i] << 16);
                        f[i + 4] -= __uint_as_float(w[i] & 0xFFFF0000u);
                    }
                }
                *reinterpret_cast<u32x4 *>(buf + place(c, tok, unit)) = w;
            }
        }
    };
    auto stage = [&](char *buf, int b) {
        const int left_k = k_hi - b * BLOCK, runs = (left_k < chunk * BLOCK ? left_k : chunk * BLOCK) / 8;
        for (int u = threadIdx.x; u < m * runs; u += THREADS) {
            const int tok = u / runs, unit = u % runs, at = row_of[tok];
            vec<T, 8> v = vec<T, 8>{};
            if (at >= 0)
                v = *reinterpret_cast<const vec<T, 8> *>(static_cast<const T *>(g.X) + at * g.ldx + b * BLOCK + unit * 8);
            prepare(buf, tok, unit, v);
        }
    };
    // a chunk of half the LDS in registers: loaded while the chunk before is
    // multiplied, prepared into the other buffer after it
    constexpr int HELD = FETCH ? (share_at<T, MT>() / 2 / (PL * 256) * 16 + THREADS - 1) / THREADS : 1;
    vec<T, 8> held[HELD];
    auto fetch = [&](int b) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int u = threadIdx.x + i * THREADS, tok = u / (chunk * 16), k = b * BLOCK + u % (chunk * 16) * 8;
            held[i] = vec<T, 8>{};
            if (tok < m && k < k_hi && row_of[tok] >= 0)
                held[i] = *reinterpret_cast<const vec<T, 8> *>(static_cast<const T *>(g.X) + row_of[tok] * g.ldx + k);
        }
    };
    auto deposit = [&](char *buf) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int u = threadIdx.x + i * THREADS, tok = u / (chunk * 16), unit = u % (chunk * 16);
            if (tok < m) prepare(buf, tok, unit, held[i]);
        }
    };

    // a set: U neighbouring blocks of the wave's NT column tiles.  The scales of
    // all of them are one load: 16 rows of a few bytes cost the address unit as
    // much as 16 rows of 64.
    struct Set {
        vec<unsigned, 4> w[U][NT];
        vec<T, U * GB> s[NT], o[NT];
    };
    const uint8_t *q_row[NT];
    const T *s_row[NT], *m_row[NT];
    auto point = [&](int pass) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int n = col0 + pass * cols + (my_n * NT + i) * 16 + (lane & 15);
            const int64_t at = (int64_t)t.e * N + (n < N ? n : N - 1);
            q_row[i] = g.Q + at * (K / 2) + 16 * h;
            s_row[i] = static_cast<const T *>(g.scales) + at * groups;
            m_row[i] = g.mins ? static_cast<const T *>(g.mins) + at * groups : nullptr;
        }
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
            x.o[i] = vec<T, U * GB>{};
            if (g.mins) x.o[i] = load_groups(m_row[i], b);
        }
    };

    // A result that was not finite, by the definition in FP64: (16 + q) x or what is taken
    // off again may have left FP32's range where s (q - 8) x does not, and an infinite
    // x made it NaN.  8192 x 8192: 0.2 to 1 ms for a row with such an entry; where there is
    // none, nothing measurable.
    auto mend = [&](int tok, int col) __attribute__((always_inline)) {
        T *const y = Y + (t.first + tok) * g.ldy + col;
        float *const p = part ? part + (t.first + tok) * N + col : nullptr;
        if (p ? isfinite(*p) : isfinite((float)*y)) return;
        const int64_t w_row = (int64_t)t.e * N + col;
        const uint8_t *const q = g.Q + w_row * (K / 2);
        const T *const s = static_cast<const T *>(g.scales) + w_row * groups;
        const T *const o = g.mins ? static_cast<const T *>(g.mins) + w_row * groups : nullptr;
        const T *const x = row_of[tok] < 0 ? nullptr : static_cast<const T *>(g.X) + row_of[tok] * g.ldx;
        double sum = 0.0;
#pragma unroll 1
        for (int k = b_lo * BLOCK; k < k_hi; k += 8) {
            const unsigned fields = (*reinterpret_cast<const vec<unsigned, 1> *>(q + k / 2))[0];
            const double scale = (float)s[k / G], offset = o ? (float)o[k / G] : 0.0f;
            vec<T, 8> v = vec<T, 8>{};
            if (x) v = *reinterpret_cast<const vec<T, 8> *>(x + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int field = fields >> (4 * i) & 15;
                sum += (o ? scale * field + offset : scale * (field - 8)) * (double)(float)v[i];
            }
        }
        if (p) *p = (float)sum;
        else *y = (T)(float)sum;
    };

    sums_t y[NT][MT] = {};
    int at[MT][4];                  // the lane's units of a block
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int want = FEW ? (lane & 15) / 4 : 16 * a + (lane & 15), tok = want < m ? want : m - 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) at[a][j] = place(0, tok, 4 * j + h);
    }
    const unsigned mask = field_mask<C>();
    frag<C> ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (C)1.0f;
    Set now, next;
    point(0);
    if (sets > 0) load(now, 0);
    __syncthreads();                                  // row_of
    if (sets > 0 && copies) copy(lds, b_lo);          // (the only chunk, or the first)
    int buf_at = ahead ? buf_bytes : 0;               // the next trip's chunk is in the other buffer
    // the sets of all passes; without any (K = 0), the passes alone
    int pass = 0, set = 0;
    do {
        if (sets > 0) {
            if (set % in_chunk == 0 && (!once || pass == 0)) {
                const int b = b_lo + set * step;
                if (FETCH && ahead) {
                    // every wave is done with the chunk before the last, whose buffer this one takes
                    if (pass + set == 0) fetch(b);
                    buf_at = buf_bytes - buf_at;
                    deposit(lds + buf_at);
                    fetch(b + chunk < b_hi ? b + chunk : b_lo);
                    __syncthreads();
                } else if (ahead) {
                    // its copies have landed, and every wave is done with the other buffer
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __syncthreads();
                    copy(lds + buf_at, b + chunk < b_hi ? b + chunk : b_lo);
                    buf_at = buf_bytes - buf_at;
                } else {
                    if (pass + set > 0) {
                        __syncthreads();              // every wave is done with the chunk before
                        if (copies) copy(lds, b);
                    }
                    if (!copies) stage(lds, b);
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __syncthreads();
                }
            }
            char *const buf = lds + buf_at;
            // the set after this one, or the next pass's first (after the last, that again)
            if (set + 1 == sets && pass + 1 < passes) point(pass + 1);
            load(next, set + 1 < sets ? set + 1 : (pass + 1 < passes ? 0 : set));
            const float *const sums = reinterpret_cast<const float *>(buf + sums_in);
            // block u of the set; whole: all of its indices are there
            auto multiply = [&](int u, auto whole) __attribute__((always_inline)) {
                const int b = block_of(set, u);
                const int in = (set % in_chunk * wk + my_k) * U + u;     // block of the chunk
                unsigned w[NT][4];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[i][j] = now.w[u][i][j];
                    exchange_quarters(w[i]);
                }
                f32x4 acc[NT][MT], xs[MT];            // xs: the sums of x (raw)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!decltype(whole)::value && b * BLOCK + 32 * j >= K) break;
                    const float *const sum = sums + (in * GB + 32 * j / G) * TOKENS + REGS * h;
                    if (32 * j % G == 0) {
#pragma unroll
                        for (int a = 0; a < MT; ++a) {
                            f32x4 c = {};
                            if constexpr (!RAW) {
                                const sums_t v = *reinterpret_cast<const sums_t *>(sum + 16 * a);
#pragma unroll
                                for (int r = 0; r < REGS; ++r) c[r] = v[r];
                            }
                            xs[a] = c;
#pragma unroll
                            for (int i = 0; i < NT; ++i) acc[i][a] = c;
                        }
                    }
                    frag<C> x[MT][PL];
#pragma unroll
                    for (int a = 0; a < MT; ++a)
#pragma unroll
                        for (int c = 0; c < PL; ++c) {
                            x[a][c] = *reinterpret_cast<const frag<C> *>(buf + at[a][j] + c * m * RB + in * 256);
                            if constexpr (RAW) x[a][c] = to_fields(x[a][c]);
                        }
                    if constexpr (RAW) {
#pragma unroll
                        for (int a = 0; a < MT; ++a) xs[a] = mfma16(x[a][0], ones, xs[a]);
                    }
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const frag<C> wf = sixteen_plus<C>(w[i][j], mask);
#pragma unroll
                        for (int c = PL - 1; c >= 0; --c)
#pragma unroll
                            for (int a = 0; a < MT; ++a) acc[i][a] = mfma16(x[a][c], wf, acc[i][a]);
                    }
                    // reads of the next run do not start before this point: no registers for more
                    if constexpr (MT > 1) __builtin_amdgcn_sched_barrier(0);
                    if ((32 * j + 32) % G == 0) {
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            const float s = (float)now.s[i][u * GB + 32 * j / G], o = (float)now.o[i][u * GB + 32 * j / G];
                            if constexpr (RAW) {      // s acc + (start s + offset) sum x
                                const float e = fmaf(start, s, o);
#pragma unroll
                                for (int a = 0; a < MT; ++a)
#pragma unroll
                                    for (int r = 0; r < REGS; ++r)
                                        y[i][a][r] = fmaf(xs[a][r], e, fmaf(acc[i][a][r], s, y[i][a][r]));
                            } else {                  // the sums are start sum x, and in acc
#pragma unroll
                                for (int a = 0; a < MT; ++a)
#pragma unroll
                                    for (int r = 0; r < REGS; ++r) y[i][a][r] = fmaf(acc[i][a][r], s, y[i][a][r]);
                                if (g.mins) {
#pragma unroll
                                    for (int a = 0; a < MT; ++a) {
                                        const sums_t v = *reinterpret_cast<const sums_t *>(sum + 16 * a);
#pragma unroll
                                        for (int r = 0; r < REGS; ++r)
                                            y[i][a][r] = fmaf(v[r], o * (1.0f / -16.0f), y[i][a][r]);
                                    }
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
            if (++set < sets) continue;
            set = 0;
        }
        // the pass's results: the lanes' own, or the sums of the waves along the reduction, in order
        const int c0 = col0 + pass * cols;
        odd = 0.0f;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            if (wk == 1) {
                const int col = c0 + (my_n * NT + i) * 16 + (lane & 15);
#pragma unroll
                for (int a = 0; a < MT; ++a)
#pragma unroll
                    for (int r = 0; r < REGS; ++r) {
                        const int tok = 16 * a + REGS * h + r;
                        if (tok < m && col < N) put(tok, col, y[i][a][r]);
                    }
            } else {
                float *const share = reinterpret_cast<float *>(lds + share_at<T, MT>());
                if (pass + i > 0) __syncthreads();
#pragma unroll
                for (int a = 0; a < MT; ++a)
#pragma unroll
                    for (int r = 0; r < REGS; ++r)
                        share[(wave * MT + a) * 256 + (REGS * h + r) * 16 + (lane & 15)] = y[i][a][r];
                __syncthreads();
                for (int j = threadIdx.x; j < m * 16 * wn; j += THREADS) {
                    const int tok = j / (16 * wn), n = j / 16 % wn, c = j % 16, col = c0 + (n * NT + i) * 16 + c;
                    if (col >= N) continue;
                    float v = 0.0f;
                    for (int w = 0; w < wk; ++w)
                        v += share[((w * wn + n) * MT + tok / 16) * 256 + tok % 16 * 16 + c];
                    put(tok, col, v);
                }
            }
#pragma unroll
            for (int a = 0; a < MT; ++a) y[i][a] = sums_t{};
        }
        if (__builtin_expect(odd != odd, 0)) {        // the thread's own results again
            const int all = m * 16 * wn, per = wk == 1 ? MT * REGS : (all + THREADS - 1) / THREADS;
#pragma unroll 1
            for (int n = 0; n < NT * per; ++n) {
                const int i = n / per, j = n % per, u = threadIdx.x + j * THREADS;
                const int tok = wk == 1 ? 16 * (j / REGS) + REGS * h + j % REGS : u / (16 * wn);
                const int of = wk == 1 ? my_n : u / 16 % wn, c = wk == 1 ? lane & 15 : u % 16;
                const int col = c0 + (of * NT + i) * 16 + c;
                if (tok < m && col < N && (wk == 1 || u < all)) mend(tok, col);
            }
        }
        ++pass;
    } while (pass < passes);
    // the last copies may not be read: they must land before the workgroup ends
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <typename T, int MT, int NT, int U, int G>
__global__ __launch_bounds__(64 * WAVES, MT == 1 && Q4Elem<T>::PLANES == 1 ? 4 : 2) void q4_gemm_kernel(Q4Gemm g,
                                                                                                         Q4Plan p) {
    __shared__ __attribute__((aligned(16))) char lds[lds_bytes<T, MT>()];
    const int cols = 16 * NT * (WAVES / p.wk) * p.passes;
    const RowTile t = RowTiles(g.offsets, g.E, g.R, 16 * MT, (g.N + cols - 1) / cols).at(blockIdx.x);
    if (t.e < 0) return;
    if (MT == 1 && t.end - t.first <= 4) q4_tile<T, MT, NT, U, G, MT == 1>(g, p, t, lds);
    else q4_tile<T, MT, NT, U, G, false>(g, p, t, lds);
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

template <typename T, int MT, int NT, int U>
Q4Plan plan_q4(const Q4Gemm &g) {
    Q4Plan p = {};
    const int tokens = g.R < 16 * MT ? (int)g.R : 16 * MT;
    const int blocks = (g.K + BLOCK - 1) / BLOCK;
    const bool once = buffer_bytes<T>(tokens, 16 * MT, g.group, blocks) <= share_at<T, MT>();
    const int bufs = Q4Elem<T>::PLANES == 1 || MT > 1 ? 2 : 1;
    int fit = once ? blocks : blocks_that_fit<T>(tokens, 16 * MT, g.group, share_at<T, MT>() / bufs);
    if (fit < U) fit = U;
    const int64_t rows = likely_tiles(g, 16 * MT);
    auto col_tiles = [&](int wk) { return (g.N + 16 * NT * (WAVES / wk) - 1) / (16 * NT * (WAVES / wk)); };
    // waves along the columns, as long as there are 16 waves for each CU
    p.wk = Q4Elem<T>::PLANES == 3 && MT > 1 ? 1 : WAVES;
    while (p.wk > 1 && ((!once && p.wk * U > fit) || rows * col_tiles(p.wk / 2) * WAVES >= 16 * 256)) p.wk /= 2;
    // few workgroups: more along the reduction, each with a set or more for its waves
    const int64_t tiles = rows * col_tiles(p.wk);
    p.splits = 1;
    while (p.splits < 16 && tiles * p.splits * 2 <= 256 && blocks / (p.splits * 2) >= 2 * p.wk * U) p.splits *= 2;
    // more workgroups than run at a time: column tiles one after the other in
    // each, so that x is staged once for them and the loads never pause
    p.passes = 1;
    while (p.passes < 16 && tiles >= 512 * 2 * p.passes) p.passes *= 2;
    return p;
}

}  // namespace

template <typename T>
int run_q4_gemm(const Q4Gemm &g, hipStream_t s) {
    int rc = EMU_OK;
    auto run = [&](auto mt, auto nt, auto set, auto group) {
        constexpr int MT = decltype(mt)::value, NT = decltype(nt)::value, U = decltype(set)::value;
        Q4Plan p = plan_q4<T, MT, NT, U>(g);
        if (p.splits > 1) {
            char *w = nullptr;
            rc = api_try_workspace(sizeof(float) * p.splits * g.R * g.N, &w);
            if (rc != EMU_OK) return;
            if (!w) p.splits = 1;       // one workgroup for the whole reduction
            p.part = reinterpret_cast<float *>(w);
        }
        p.copies = reinterpret_cast<uintptr_t>(g.X) % 16 == 0 && g.ldx % 8 == 0;
        const int cols = 16 * NT * (WAVES / p.wk) * p.passes;
        const int64_t tiles = row_blocks_bound(g.R, g.E, 16 * MT) * ((g.N + cols - 1) / cols);
        q4_gemm_kernel<T, MT, NT, U, decltype(group)::value><<<dim3((unsigned)tiles, p.splits), 64 * WAVES, 0, s>>>(g, p);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && p.splits > 1) {
            q4_join_kernel<T><<<(unsigned)((g.R * g.N + 255) / 256), 256, 0, s>>>(p.part, p.splits, g.R, g.N,
                                                                                  static_cast<T *>(g.Y), g.ldy);
            e = hipGetLastError();
        }
        rc = api_done(e, "q4_gemm");
    };
    auto rows = [&](auto group) {
        using std::integral_constant;
        const integral_constant<int, 1> one;
        const integral_constant<int, 2> two;
        const integral_constant<int, 3> three;
        const integral_constant<int, 4> four;
        // A wave has 4 KB of weights in flight, 2 KB where the accumulators leave no
        // registers for more (float32, and tiles of 64).  Two column tiles to a wave above
        // 16 rows: with four, 40 half rows of 8192 x 8192 took 64 us instead of 40 (spills).
        // Above 48 float32 rows tiles of 32, whose weights are read twice: 64 rows of
        // 4096 x 8192 take 40 us, a tile of 64, which spills, 95.
        constexpr bool wide = Q4Elem<T>::PLANES == 3;
        const integral_constant<int, wide ? 1 : 2> set;
        const int tile = q4_tile_rows(g.dtype, g.R, g.E > 0 ? g.E : 1);
        if (tile == 16) run(one, one, four, group);
        else if (tile == 32) run(two, two, set, group);
        else if (tile == 48) run(three, two, set, group);
        else if constexpr (!wide) run(four, two, one, group);
    };
    if (g.group == 32) rows(std::integral_constant<int, 32>{});
    else if (g.group == 64) rows(std::integral_constant<int, 64>{});
    else rows(std::integral_constant<int, 128>{});
    return rc;
}

}  // namespace emu
