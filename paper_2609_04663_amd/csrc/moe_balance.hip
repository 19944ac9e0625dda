// The balance loss of a routing, for each sequence of tokens, and its gradient.
//
// With p the softmax of a token's logits over all experts, z the logarithm of its sum,
// n the tokens of the sequence that have a logit above -inf and c_e the choices of
// expert e, C of them in all:
//   loss = E sum_e (c_e / C) (1 / n) sum_t p[t, e]      zloss = (1 / n) sum_t z[t]^2
//   d/dlogits[t, e] = p[t, e] (dloss E / n (f_e - sum_j p_j f_j) + dzloss 2 / n z[t]),
// f_e = c_e / C, which is taken as constant.  LANES lanes hold a token's logits in
// registers, four neighbouring ones in a load.
//
// A workgroup sums a span of one sequence's tokens: the probabilities in registers over
// the tokens of a group of lanes, over the groups in LDS, the counts by integer atomics
// there; another kernel joins a sequence's spans in FP64, in order, so no atomic decides
// a sum.  Which span a workgroup has is known on the device only: sequence s starts at
// workgroup first token / span + s, which leaves room for every span before it, so a
// search in the starts finds it.  Few tokens take one workgroup a sequence and one launch.
//
// Measured: 64 tokens of 64 experts 4.2 us; 16384 bfloat16 tokens of 128 experts 6 + 7 us, the
// gradient 7; 65536 float32 tokens of 256 experts in 33 sequences 18 + 6 us (the first 3.9 TB/s),
// the gradient 29 to 31 (4.4 TB/s).
#include "api_state.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int64_t ONE_LAUNCH = 256;         // tokens

// Workgroup `id`'s tokens [first, end) of sequence s, s == S: of none.
struct Span {
    int s;
    int64_t first, end;
};
// By whole waves: 64 candidates at a time.
__device__ inline Span span_of(const int *__restrict__ starts, int S, int64_t T, int span, int64_t id) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = S;
    int64_t first, end;
    while (lo < hi) {
        const int step = (hi - lo + 64) / 64, s = lo + lane * step;
        bool from = false;
        if (s <= hi) {
            expert_rows(starts, S, T, s, first, end);
            from = (int)first / span + s <= id;
        }
        const unsigned long long all = __ballot(from || lane == 0);
        lo += (63 - __builtin_clzll(all)) * step;
        hi = lo + step - 1 < hi ? lo + step - 1 : hi;
    }
    lo = uniform(lo);
    expert_rows(starts, S, T, lo, first, end);
    const int64_t at = first + (id - (int)first / span - lo) * span;
    if (at >= end) return {lo, end, end};
    return {lo, at, at + span < end ? at + span : end};
}

// Where the joining kernel finds a workgroup's sums: E probabilities and E counts, each in
// a row of a multiple of four, then the sum of z^2 (FP64) and the tokens.
__host__ __device__ constexpr int padded(int E) { return (E + 3) & ~3; }
__host__ __device__ constexpr int64_t sums_of(int E) { return 2 * padded(E) + 4; }

// The logits of a token in LANES lanes: x[4 c + j] is expert 4 (c LANES + sub) + j, -inf
// past the last and for NaN.
template <int LANES, int V, typename T>
__device__ __forceinline__ void load_token(const T *__restrict__ row, int E, int sub, float (&x)[V]) {
#pragma unroll
    for (int c = 0; c < V / 4; ++c) {
        const int e = (c * LANES + sub) * 4;
        if (e + 4 <= E) {
            const vec<T, 4> v = *reinterpret_cast<const vec<T, 4> *>(row + e);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * c + j] = fmaxf((float)v[j], -INFINITY);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * c + j] = e + j < E ? fmaxf((float)row[e + j], -INFINITY) : -INFINITY;
        }
    }
}

// x becomes the probabilities (zeros where no logit is above -inf); returns the logarithm
// of the softmax's sum, *live whether there is a logit.  exp(d) for d = x - m <= 0 is the
// hardware's 2^(d log2 e): off by |d| 2^-24 for the product's rounding and as much for that
// of d, so by what d itself is uncertain by.  With the library's expf, which takes the
// product's rounding back, the loss of 65536 tokens and 256 experts took 34 us instead of 26.
template <int LANES, int V>
__device__ __forceinline__ float softmax(float (&x)[V], bool *live) {
    constexpr float LOG2E = 1.44269504f;
    float m = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) m = fmaxf(m, x[i]);
    m = over_lanes<LANES>(m, [](float a, float b) { return fmaxf(a, b); });
    *live = m > -INFINITY;
    float from = *live ? m : 0.0f;
    if (m == INFINITY) {                                    // its experts share the weight
        from = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = x[i] == INFINITY ? 0.0f : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = __builtin_amdgcn_exp2f((x[i] - from) * LOG2E);
        sum += x[i];
    }
    sum = over_lanes<LANES>(sum, [](float a, float b) { return a + b; });
    const float scale = *live ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= scale;
    return *live ? m + logf(sum) : 0.0f;
}

__device__ __forceinline__ double over_wave(double v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A sequence's results from the sums of expert e = threadIdx.x: of probabilities and of
// choices (zeros past the last expert); z and n in thread 0.
__device__ inline void finish(int E, int s, double p, int c, double z, int n, float *__restrict__ loss,
                              float *__restrict__ zloss, int *__restrict__ counts, int *__restrict__ tokens) {
    __shared__ double dot[WAVES], all[WAVES];
    const int e = threadIdx.x, wave = e >> 6;
    if (e < E) counts[(int64_t)s * E + e] = c;
    const double d = over_wave(p * c), a = over_wave((double)c);
    if ((e & 63) == 0) {
        dot[wave] = d;
        all[wave] = a;
    }
    __syncthreads();
    if (e == 0) {
        double sum = 0, choices = 0;
        for (int w = 0; w < WAVES; ++w) {
            sum += dot[w];
            choices += all[w];
        }
        loss[s] = n > 0 && choices > 0 ? (float)(E * sum / (choices * n)) : 0.0f;
        zloss[s] = n > 0 ? (float)(z / n) : 0.0f;
        tokens[s] = n;
    }
}

// span 0: a workgroup for each sequence, whose results it writes; else the sums go to `sums`.
// Two workgroups to a CU (8 waves to a SIMD) where the registers allow it, which hide the
// loads better than loads ahead in more registers: 18 us for 65536 tokens and 256 experts
// in 33 sequences (3.9 TB/s) instead of 26.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(THREADS, V <= 16 ? 8 : 4) void balance_kernel(BalanceLoss b, int span, float *__restrict__ sums) {
    __shared__ float part[WAVES][LANES * V];
    __shared__ int count[ROUTE_EXPERTS], n_of[WAVES];
    __shared__ double z_of[WAVES];
    constexpr int GROUPS = THREADS / LANES;
    const int tid = threadIdx.x, sub = tid % LANES, lane = tid & 63, wave = tid >> 6, E = b.E;
    Span at;
    if (span > 0) {
        at = span_of(b.starts, b.S, b.T, span, blockIdx.x);
        if (at.s == b.S || at.first == at.end) return;
    } else {
        at.s = blockIdx.x;
        expert_rows(b.starts, b.S, b.T, at.s, at.first, at.end);
    }
    count[tid] = 0;
    __syncthreads();
    const T *const logits = static_cast<const T *>(b.logits);
    const int64_t last = at.end - 1;
    float acc[V] = {};
    double z = 0;                                           // FP32 does not hold the squares of all z
    int n = 0;
    int64_t t = at.first + tid / LANES;
    for (int64_t i = tid, choices = (at.end - at.first) * b.k; i < choices; i += THREADS) {
        const int e = b.ids[at.first * b.k + i];
        if (e >= 0 && e < E) atomicAdd(&count[e], 1);
    }
    for (int64_t t0 = at.first; t0 < at.end; t0 += GROUPS, t += GROUPS) {
        float x[V];
        bool live;
        load_token<LANES, V>(logits + (t < last ? t : last) * b.ld, E, sub, x);
        const float lse = softmax<LANES, V>(x, &live);
        if (t > last) continue;                             // the group's last load stands in
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += x[i];
        z += (double)lse * lse;
        n += live;
    }
    // over the groups of the wave, then over the waves
#pragma unroll
    for (int d = LANES; d < 64; d <<= 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += __shfl_xor(acc[i], d);
        z += __shfl_xor(z, d);
        n += __shfl_xor(n, d);
    }
    if (lane < LANES)
#pragma unroll
        for (int i = 0; i < V; ++i) part[wave][(i / 4 * LANES + sub) * 4 + i % 4] = acc[i];
    if (lane == 0) {
        z_of[wave] = z;
        n_of[wave] = n;
    }
    __syncthreads();
    double p = 0, zs = 0;
    int ns = 0;
    if (tid < E)
        for (int w = 0; w < WAVES; ++w) p += part[w][tid];
    if (tid == 0)
        for (int w = 0; w < WAVES; ++w) {
            zs += z_of[w];
            ns += n_of[w];
        }
    if (span == 0) {
        finish(E, at.s, p, tid < E ? count[tid] : 0, zs, ns, b.loss, b.zloss, b.counts, b.tokens);
        return;
    }
    float *const out = sums + blockIdx.x * sums_of(E);
    if (tid < padded(E)) {                                  // zeros past the last expert
        out[tid] = (float)p;
        out[padded(E) + tid] = __int_as_float(tid < E ? count[tid] : 0);
    }
    if (tid == 0) {
        *reinterpret_cast<double *>(out + 2 * padded(E)) = zs;
        out[2 * padded(E) + 2] = __int_as_float(ns);
    }
}

// A workgroup joins the spans of its sequence: a thread has four neighbouring experts, W
// threads (the power of two from E / 4 on) all of them, of 1024 / W spans at a time; the
// loads of AHEAD of these in flight (one expert to a thread and four loads ahead: 15 us
// instead of 7 for 256 spans of 128 experts, which one workgroup reads where there is one sequence).
__global__ __launch_bounds__(THREADS) void balance_join_kernel(BalanceLoss b, int span, int W,
                                                               const float *__restrict__ sums) {
    __shared__ double p_of[THREADS][4], z_of[WAVES];
    __shared__ int c_of[THREADS][4], n_of[WAVES];
    constexpr int AHEAD = 8;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const int tid = threadIdx.x, e = (tid & (W - 1)) * 4, E = b.E, s = blockIdx.x, G = THREADS / W;
    int64_t first, end;
    expert_rows(b.starts, b.S, b.T, s, first, end);
    const int spans = (int)((end - first + span - 1) / span);
    const int64_t stride = sums_of(E);
    const float *const from = sums + ((int)first / span + s) * stride;
    double p[4] = {}, z = 0;
    int c[4] = {}, n = 0;
    for (int i = tid; i < spans; i += THREADS) {
        const float *const last = from + i * stride + 2 * padded(E);
        z += *reinterpret_cast<const double *>(last);
        n += __float_as_int(last[2]);
    }
    if (e < E)
        for (int i0 = tid / W; i0 < spans; i0 += AHEAD * G) {
            f32x4 ps[AHEAD], cs[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int i = i0 + a * G < spans ? i0 + a * G : i0;
                ps[a] = *reinterpret_cast<const f32x4 *>(from + i * stride + e);
                cs[a] = *reinterpret_cast<const f32x4 *>(from + i * stride + padded(E) + e);
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a)
                if (i0 + a * G < spans)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        p[j] += ps[a][j];
                        c[j] += __float_as_int(cs[a][j]);
                    }
        }
    z = over_wave(z);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
    if ((tid & 63) == 0) {
        z_of[tid >> 6] = z;
        n_of[tid >> 6] = n;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        p_of[tid][j] = p[j];
        c_of[tid][j] = c[j];
    }
    __syncthreads();
    double sum = 0;
    int count = 0;
    if (tid < E)
        for (int g = 0; g < G; ++g) {
            sum += p_of[g * W + tid / 4][tid & 3];
            count += c_of[g * W + tid / 4][tid & 3];
        }
    z = 0;
    n = 0;
    for (int w = 0; w < WAVES; ++w) {
        z += z_of[w];
        n += n_of[w];
    }
    finish(E, s, sum, count, z, n, b.loss, b.zloss, b.counts, b.tokens);
}

template <typename T, int LANES, int V>
__global__ __launch_bounds__(256) void balance_grad_kernel(BalanceGrad b, int span) {
    constexpr int GROUPS = 256 / LANES;
    const int tid = threadIdx.x, sub = tid % LANES, E = b.E;
    const Span at = span_of(b.starts, b.S, b.T, span, blockIdx.x);
    if (at.first == at.end) return;
    const bool none = at.s == b.S;
    const int s = none ? 0 : at.s;
    const T *const logits = static_cast<const T *>(b.logits);
    T *const out = static_cast<T *>(b.dlogits);
    const int64_t last = at.end - 1;
    int64_t t = at.first + tid / LANES;
    float next[V], f[V], choices = 0.0f;
    load_token<LANES, V>(logits + (t < last ? t : last) * b.ld, E, sub, next);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = (i / 4 * LANES + sub) * 4 + i % 4;
        f[i] = e < E ? (float)b.counts[(int64_t)s * E + e] : 0.0f;
        choices += f[i];
    }
    choices = over_lanes<LANES>(choices, [](float a, float b) { return a + b; });
    const int n = none ? 0 : b.tokens[s];
    // (a token's share first: dloss E may leave FP32's range where dloss E / n does not)
    const float per = n > 0 ? 1.0f / n : 0.0f, dl = n > 0 ? b.dloss[s] * (E * per) : 0.0f;
    const float dz = n > 0 && b.dzloss ? b.dzloss[s] * (2.0f * per) : 0.0f;
    const float share = choices > 0.0f ? 1.0f / choices : 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] *= share;
    for (int64_t t0 = at.first; t0 < at.end; t0 += GROUPS, t += GROUPS) {
        float x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = next[i];
        const int64_t ahead = t + GROUPS < last ? t + GROUPS : last;
        if (t0 + GROUPS < at.end) load_token<LANES, V>(logits + ahead * b.ld, E, sub, next);
        bool live;
        const float lse = softmax<LANES, V>(x, &live);
        float mean = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) mean += x[i] * f[i];
        mean = over_lanes<LANES>(mean, [](float a, float b) { return a + b; });
        if (t > last) continue;
        // an infinite z concerns the experts that share the weight, the others stay 0
        const float shift = dz != 0.0f ? dz * lse : 0.0f;
        T *const row = out + t * b.ldd;
#pragma unroll
        for (int c = 0; c < V / 4; ++c) {
            const int e = (c * LANES + sub) * 4;
            float g[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = x[4 * c + j];
                g[j] = p > 0.0f && n > 0 ? p * (dl * (f[4 * c + j] - mean) + shift) : 0.0f;
            }
            if (e + 4 <= E) {
                store_f32<4>(row + e, g);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (e + j < E) row[e + j] = (T)g[j];
            }
        }
    }
}

// f(lanes, values of a lane) for E experts.
template <typename F>
void with_shape(int E, F &&f) {
    using std::integral_constant;
    const integral_constant<int, 16> sixteen;
    if (E <= 16) f(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    else if (E <= 64) f(sixteen, integral_constant<int, 4>{});
    else if (E <= 128) f(sixteen, integral_constant<int, 8>{});
    else if (E <= 256) f(sixteen, sixteen);
    else if (E <= 512) f(sixteen, integral_constant<int, 32>{});
    else f(integral_constant<int, 64>{}, sixteen);
}

// Tokens of a workgroup: some 448 workgroups, so that they and those of the sequences' last
// spans are on the chip at a time, and the joining kernel has few spans to read.
int span_of_sums(int64_t T) {
    constexpr int64_t WORKGROUPS = 448;
    const int64_t n = (T + WORKGROUPS - 1) / WORKGROUPS;
    return (int)(n <= 64 ? 64 : (n + 63) / 64 * 64);
}

}  // namespace

size_t balance_scratch(int64_t T, int E, int S) {
    return T <= ONE_LAUNCH ? 0 : (T / span_of_sums(T) + S) * sums_of(E) * sizeof(float);
}

hipError_t launch_balance(const BalanceLoss &b, char *scratch, hipStream_t s) {
    const int span = b.T <= ONE_LAUNCH ? 0 : span_of_sums(b.T);
    const unsigned grid = span ? (unsigned)(b.T / span + b.S) : b.S;
    float *const sums = reinterpret_cast<float *>(scratch);
    with_type(b.dtype, [&](auto z) {
        using T = decltype(z);
        with_shape(b.E, [&](auto lanes, auto v) {
            balance_kernel<T, decltype(lanes)::value, decltype(v)::value><<<grid, THREADS, 0, s>>>(b, span, sums);
        });
    });
    hipError_t e = hipGetLastError();
    if (span == 0 || e != hipSuccess) return e;
    int W = 1;
    while (4 * W < b.E) W *= 2;
    balance_join_kernel<<<b.S, THREADS, 0, s>>>(b, span, W, sums);
    return hipGetLastError();
}

hipError_t launch_balance_grad(const BalanceGrad &b, hipStream_t s) {
    with_type(b.dtype, [&](auto z) {
        using T = decltype(z);
        with_shape(b.E, [&](auto lanes, auto v) {
            // some 2048 workgroups at most; the tokens of no sequence among them
            constexpr int LANES = decltype(lanes)::value, GROUPS = 256 / LANES;
            const int span = (int)((b.T + 2048 * GROUPS - 1) / (2048 * GROUPS)) * GROUPS;
            const unsigned grid = (unsigned)(b.T / span + b.S + 1);
            balance_grad_kernel<T, LANES, decltype(v)::value><<<grid, 256, 0, s>>>(b, span);
        });
    });
    return hipGetLastError();
}

}  // namespace emu
