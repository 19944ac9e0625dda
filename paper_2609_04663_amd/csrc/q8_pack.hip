// Rows in 8-bit integers with one scale each, and back.
//
// With top = max |x| of a row: scale = top / 127, q = the integer nearest 127 x / top,
// ties to even.  A row of zeros has scale 0, one with an infinity or a NaN the scale NaN
// and zeros, so that everything made from it is NaN.
//
// x inv + 1.5 2^23 with inv = 127 / top, one fused multiply-add, has the integer nearest
// x inv in its low bits.  inv is off by half a unit in its last place, so x inv by at most
// 127 2^-24 < 2^-17, and where it lies nearer than that to a border between two integers
// they are compared in FP64, in which 127 x and n top (31 bits) are exact.
//
// One pass: LANES lanes hold a row in registers, eight entries in a load (longer rows are
// read a second time).  Bound by bytes: 131072 bfloat16 rows of 2048 in 157 us (5.1 TB/s), back
// in 127 (6.3 TB/s, the integers partly from the last-level cache); one row of 4096 2.3 us.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int UNIT = 8;                                 // entries of a load

template <typename T>
using unit = T __attribute__((ext_vector_type(UNIT)));

// A lane takes the entries e .. e + 7 of a row of K.  Where the row ends in between, or
// before, it takes the row's last eight: entries that another lane has too, and both make
// the same of them (so no lane has a path of its own: 4999 float32 rows of 1501 12 -> 9 us).
// Rows of fewer than eight are read one by one, zeros behind them.
__device__ __forceinline__ int place_of(int e, int K) { return e + UNIT <= K || K < UNIT ? e : K - UNIT; }
template <typename T>
__device__ __forceinline__ unit<T> load_unit(const T *__restrict__ row, int e, int K) {
    if (K >= UNIT) return *reinterpret_cast<const vec<T, UNIT> *>(row + place_of(e, K));
    unit<T> v = unit<T>{};
#pragma unroll
    for (int j = 0; j < UNIT; ++j)
        if (e + j < K) v[j] = row[e + j];
    return v;
}

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

template <typename T>
__device__ __forceinline__ unsigned top_of(unit<T> v) {
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < UNIT; ++j) {
        const unsigned m = magnitude((float)v[j]);     // as integers: NaN above infinity
        top = m > top ? m : top;
    }
    return top;
}

// How a row is brought to integers: top and the entries are taken times `up`, which keeps
// inv and the products normal where the row is tiny.
struct Row {
    float top, inv, up;
    __device__ __forceinline__ Row(unsigned bits, float *scale, bool writes) {
        const bool finite = bits < 0x7F800000u;
        top = finite ? __uint_as_float(bits) : 0.0f;
        if (writes) *scale = finite ? top / 127.0f : NAN;
        up = top < 0x1p-60f ? 0x1p64f : 1.0f;
        top *= up;
        inv = top > 0.0f ? 127.0f / top : 0.0f;
    }
};

template <typename T>
__device__ __forceinline__ uint2 quantise(unit<T> v, const Row &r) {
    constexpr float ROUND = 0x1.8p23f;
    float x[UNIT], u[UNIT], off = 0.0f;
#pragma unroll
    for (int j = 0; j < UNIT; ++j) {
        x[j] = (float)v[j] * r.up;
        u[j] = __builtin_fmaf(x[j], r.inv, ROUND);
        off = fmaxf(off, fabsf(__builtin_fmaf(x[j], r.inv, -(u[j] - ROUND))));
    }
    if (r.top == 0.0f) return {0, 0};                   // zeros, or not finite
    unsigned q[UNIT];
#pragma unroll
    for (int j = 0; j < UNIT; ++j) q[j] = __float_as_uint(u[j]);
    if (off > 0.5f - 0x1p-16f) {                        // one of them is at a border
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            const float n = u[j] - ROUND;
            const double rest = 127.0 * x[j] - (double)n * r.top, half_top = 0.5 * r.top;
            const bool odd = (q[j] & 1) != 0;
            if (rest > half_top || (rest == half_top && odd)) q[j] += 1;
            else if (rest < -half_top || (rest == -half_top && odd)) q[j] -= 1;
        }
    }
    uint2 w;
    w.x = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | q[3] << 24;
    w.y = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | q[7] << 24;
    return w;
}

__device__ __forceinline__ void store_unit(int8_t *__restrict__ row, int e, int K, uint2 w) {
    typedef unsigned __attribute__((ext_vector_type(2), aligned(1))) u32x2;
    if (K >= UNIT) {
        *reinterpret_cast<u32x2 *>(row + place_of(e, K)) = u32x2{w.x, w.y};
    } else {
#pragma unroll
        for (int j = 0; j < UNIT; ++j)
            if (e + j < K) row[e + j] = (int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
}

__device__ __forceinline__ unsigned max_of(unsigned a, unsigned b) { return a > b ? a : b; }

constexpr int64_t MOST = (1 << 24) - 8;                 // workgroups of a launch

// LANES lanes to a row, 256 / LANES rows to a workgroup; UNITS of eight entries to a lane,
// 0: as many as there are, read twice.
template <typename T, int LANES, int UNITS>
__global__ __launch_bounds__(256) void q8_pack_kernel(const T *__restrict__ X, int64_t rows, int64_t ldx, int K,
                                                      int8_t *__restrict__ Q, int64_t ldq,
                                                      float *__restrict__ scales) {
    constexpr int ROWS = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < rows; row0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = row0 + threadIdx.x / LANES;
        const bool there = row < rows;
        const T *const x = X + (there ? row : row0) * ldx;
        unit<T> v[UNITS > 0 ? UNITS : 1];
        unsigned top = 0;
        if constexpr (UNITS > 0) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) v[i] = load_unit(x, (i * LANES + lane) * UNIT, K);
#pragma unroll
            for (int i = 0; i < UNITS; ++i) top = max_of(top, top_of<T>(v[i]));
        } else {
            for (int e = lane * UNIT; e < K; e += LANES * UNIT) top = max_of(top, top_of<T>(load_unit(x, e, K)));
        }
        top = over_lanes<(LANES < 64 ? LANES : 64)>(top, max_of);
        if constexpr (LANES > 64) {
            __shared__ unsigned of_wave[4];
            __syncthreads();
            if (lane % 64 == 0) of_wave[lane / 64] = top;
            __syncthreads();
            top = max_of(max_of(of_wave[0], of_wave[1]), max_of(of_wave[2], of_wave[3]));
        }
        if (!there) break;
        const Row r(top, scales + row, lane == 0);
        int8_t *const q = Q + row * ldq;
        if constexpr (UNITS > 0) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int e = (i * LANES + lane) * UNIT;
                if (e < K) store_unit(q, e, K, quantise<T>(v[i], r));
            }
        } else {
            for (int e = lane * UNIT; e < K; e += LANES * UNIT)
                store_unit(q, e, K, quantise<T>(load_unit(x, e, K), r));
        }
    }
}

// 64 lanes to a row's columns, `run` of them from blockIdx.y run on.  One unit of a lane at
// a time, and its load behind a branch, so that it stays there: with four in flight 131072
// rows of 2048 took 184 us instead of 127, with the next one's load moved up 143.
template <typename T>
__global__ __launch_bounds__(256) void q8_unpack_kernel(const int8_t *__restrict__ Q, int64_t rows, int64_t ldq,
                                                        int K, int run, const float *__restrict__ scales,
                                                        T *__restrict__ X, int64_t ldx) {
    for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; row < rows; row += (int64_t)gridDim.x * 4) {
        const float scale = scales[row];
        const int8_t *const q = Q + row * ldq;
        T *const x = X + row * ldx;
        for (int c0 = blockIdx.y * run; c0 < K; c0 += gridDim.y * run)
#pragma unroll 1
            for (int e = c0 + threadIdx.x % 64 * UNIT; e < K && e < c0 + run; e += 64 * UNIT) {
                unit<int8_t> v;
                if (e + UNIT <= K) v = *reinterpret_cast<const vec<int8_t, UNIT> *>(q + e);
                else v = load_unit(q, e, K);
                float f[UNIT];
#pragma unroll
                for (int j = 0; j < UNIT; ++j) f[j] = (float)v[j] * scale;
                if (K >= UNIT) {
                    store_f32<UNIT>(x + place_of(e, K), f);
                } else {
#pragma unroll
                    for (int j = 0; j < UNIT; ++j)
                        if (e + j < K) x[e + j] = (T)f[j];
                }
            }
    }
}

}  // namespace

hipError_t launch_q8_pack(int dtype, const void *X, int64_t rows, int64_t ldx, int64_t K, int8_t *Q, int64_t ldq,
                          float *scales, hipStream_t s) {
    with_type(dtype, [&](auto z) {
        using T = decltype(z);
        auto run = [&](auto lanes, auto units) {
            constexpr int LANES = decltype(lanes)::value, ROWS = 256 / LANES;
            const int64_t grid = (rows + ROWS - 1) / ROWS;
            q8_pack_kernel<T, LANES, decltype(units)::value><<<(unsigned)(grid < MOST ? grid : MOST), 256, 0, s>>>(
                static_cast<const T *>(X), rows, ldx, (int)K, Q, ldq, scales);
        };
        using std::integral_constant;
        const integral_constant<int, 16> sixteen;
        const integral_constant<int, 64> wave;
        const integral_constant<int, 256> group;
        const integral_constant<int, 1> one;
        const integral_constant<int, 2> two;
        const integral_constant<int, 4> four;
        const integral_constant<int, 8> eight;
        if (K <= 128) run(sixteen, one);
        else if (K <= 256) run(sixteen, two);
        else if (K <= 512) run(wave, one);
        else if (K <= 1024) run(wave, two);
        else if (K <= 2048) run(wave, four);
        else if (K <= 4096) run(group, two);
        else if (K <= 8192) run(group, four);
        else if (K <= 16384) run(group, eight);
        else run(group, integral_constant<int, 0>{});
    });
    return hipGetLastError();
}

hipError_t launch_q8_unpack(int dtype, const int8_t *Q, int64_t rows, int64_t ldq, int64_t K, const float *scales,
                            void *X, int64_t ldx, hipStream_t s) {
    // long runs of a row, but where so few workgroups would leave the chip empty
    const int64_t high = (rows + 3) / 4;
    const int run = high * ((K + 4095) / 4096) < 1024 ? 512 : 4096;
    const int64_t cols = (K + run - 1) / run, y = cols < 32768 ? cols : 32768, most = MOST / y;
    const dim3 grid((unsigned)(high < most ? high : most), (unsigned)y);
    with_type(dtype, [&](auto z) {
        using T = decltype(z);
        q8_unpack_kernel<T><<<grid, 256, 0, s>>>(Q, rows, ldq, (int)K, run, scales, static_cast<T *>(X), ldx);
    });
    return hipGetLastError();
}

}  // namespace emu
