// The weighted sum of the experts' rows of each token, y[t] = sum_j w[t, j]
// z[slots[t, j]], and its gradients, dz[slots[t, j]] = w[t, j] dy[t] and
// dw[t, j] = <z[slots[t, j]], dy[t]>.  Sums are held in 32 bits.  Bound by
// bytes: every row of z is read once (and of dz written once), 16 bytes a
// thread; a token's k rows are independent loads in flight together.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

// n <= N elements at p as floats (zeros past n)
template <int N, typename T>
__device__ __forceinline__ void load_some(const T *p, int64_t n, float (&x)[N]) {
    if (n >= N) {
        load_f32<N>(p, x);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < n ? (float)p[i] : 0.0f;
    }
}
template <int N, typename T>
__device__ __forceinline__ void store_some(T *p, int64_t n, const float (&x)[N]) {
    if (n >= N) {
        store_f32<N>(p, x);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = (T)x[i];
    }
}

// A thread takes 16 bytes of one token, AHEAD rows of z in flight; the grid is (tokens,
// chunks of D).
template <typename T, int AHEAD>
__global__ __launch_bounds__(256) void combine_kernel(const T *__restrict__ Z, int64_t ldz, int64_t R,
                                                      int64_t D, int k, const int *__restrict__ slots,
                                                      const float *__restrict__ weights,
                                                      T *__restrict__ Y, int64_t ldy) {
    constexpr int N = 16 / sizeof(T);
    const int64_t t = blockIdx.x, step = (int64_t)gridDim.y * blockDim.x * N;
    for (int64_t d = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * N; d < D; d += step) {
        float y[N] = {};
        for (int j0 = 0; j0 < k; j0 += AHEAD) {
            vec<T, N> z[AHEAD];
            float w[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int64_t at = j0 + j < k ? slots[t * k + j0 + j] : -1;
                const bool there = at >= 0 && at < R;
                w[j] = there ? (weights ? weights[t * k + j0 + j] : 1.0f) : 0.0f;
                z[j] = vec<T, N>{};
                if (there) {
                    const T *const p = Z + at * ldz + d;
                    if (d + N <= D) {
                        z[j] = *reinterpret_cast<const vec<T, N> *>(p);
                    } else {
#pragma unroll
                        for (int i = 0; i < N; ++i) z[j][i] = d + i < D ? p[i] : T(0);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) y[i] = fmaf(w[j], (float)z[j][i], y[i]);
        }
        store_some<N>(Y + t * ldy + d, D - d, y);
    }
}

// A workgroup takes a token: its dy stays in registers across the choices, four
// of which are in flight at a time.  It also clears the rows t, t + groups, ... of dz
// that belong to no token.
template <typename T>
__global__ __launch_bounds__(256) void combine_grad_kernel(
    const T *__restrict__ dY, int64_t lddy, const T *__restrict__ Z, int64_t ldz, int64_t R,
    int64_t groups, int64_t D, int k, const int *__restrict__ slots, const float *__restrict__ weights,
    const int *__restrict__ rows, T *__restrict__ dZ, int64_t lddz, float *__restrict__ dweights) {
    constexpr int N = 16 / sizeof(T);
    __shared__ float part[ROUTE_CHOICES][4];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int j0 = 0; j0 < k; j0 += 4) {
        float dot[4] = {}, w[4];
        int64_t at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            at[j] = j0 + j < k ? slots[t * k + j0 + j] : -1;
            if (at[j] >= R) at[j] = -1;
            w[j] = at[j] >= 0 ? weights[t * k + j0 + j] : 0.0f;
        }
        for (int64_t d = threadIdx.x * N; d < D; d += 256 * N) {
            float dy[N];
            load_some<N>(dY + t * lddy + d, D - d, dy);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (at[j] < 0) continue;
                float z[N], dz[N];
                load_some<N>(Z + at[j] * ldz + d, D - d, z);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dot[j] = fmaf(z[i], dy[i], dot[j]);
                    dz[i] = w[j] * dy[i];
                }
                store_some<N>(dZ + at[j] * lddz + d, D - d, dz);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int s = 32; s > 0; s >>= 1) dot[j] += __shfl_xor(dot[j], s);
            if (lane == 0) part[j0 + j][wave] = dot[j];
        }
    }
    for (int64_t r = t; r < R; r += groups) {
        if (rows[r] >= 0) continue;
        const float zero[N] = {};
        for (int64_t d = threadIdx.x * N; d < D; d += 256 * N)
            store_some<N>(dZ + r * lddz + d, D - d, zero);
    }
    __syncthreads();
    if ((int)threadIdx.x < k) {
        const float *p = part[threadIdx.x];
        dweights[t * k + threadIdx.x] = (p[0] + p[1]) + (p[2] + p[3]);
    }
}

}  // namespace

hipError_t launch_combine(int dtype, const void *Z, int64_t ldz, int64_t R, int64_t T, int64_t D,
                          int k, const int *slots, const float *weights, void *Y, int64_t ldy,
                          hipStream_t s) {
    with_type(dtype, [&](auto z) {
        using type = decltype(z);
        const int64_t chunks = (D + 16 / sizeof(type) - 1) / (16 / sizeof(type));
        const int threads = chunks <= 64 ? 64 : (chunks <= 128 ? 128 : 256);
        const int64_t parts = (chunks + threads - 1) / threads;
        const dim3 grid((unsigned)T, (unsigned)(parts < 65535 ? parts : 65535));
        auto run = [&](auto ahead) {
            combine_kernel<type, ahead><<<grid, threads, 0, s>>>(static_cast<const type *>(Z), ldz, R, D, k, slots,
                                                                 weights, static_cast<type *>(Y), ldy);
        };
        if (k <= 4) run(std::integral_constant<int, 4>{});
        else run(std::integral_constant<int, 8>{});
    });
    return hipGetLastError();
}

hipError_t launch_combine_grad(int dtype, const void *dY, int64_t lddy, const void *Z, int64_t ldz,
                               int64_t R, int64_t T, int64_t D, int k, const int *slots,
                               const float *weights, const int *rows, void *dZ, int64_t lddz,
                               float *dweights, hipStream_t s) {
    with_type(dtype, [&](auto z) {
        using type = decltype(z);
        // no tokens: workgroups without choices clear the rows
        const int64_t groups = T > 0 ? T : (R < 4096 ? R : 4096);
        combine_grad_kernel<type><<<(unsigned)groups, 256, 0, s>>>(
            static_cast<const type *>(dY), lddy, static_cast<const type *>(Z), ldz, R, groups, D, T > 0 ? k : 0,
            slots, weights, rows, static_cast<type *>(dZ), lddz, dweights);
    });
    return hipGetLastError();
}

}  // namespace emu
