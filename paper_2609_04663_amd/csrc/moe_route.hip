// The router of a mixture of experts: each token's k experts with their
// weights, the gradient of the logits, and the order of the rows by expert.
//
// Choice.  The k largest logits of a token in descending order, the lowest
// index of equal ones first; -inf and NaN are never chosen.  With m the largest
// logit, weights_j = exp(l_j - m) / sum exp(l - m), the sum over the chosen
// experts or over all (a largest logit of +inf shares the weight among the
// experts that have it).  Sixteen lanes hold a token's logits in registers, 32
// values each at most (64 lanes above 512 experts: 16 lanes take a quarter of the
// instructions, 4096 tokens and 512 experts 42 us with 64 lanes and 21 with 16); a round
// takes the largest ordered bit pattern of the lanes, then the lowest index that has
// it, each four moves between registers (through LDS they took 2 us more of a launch).
// Logits of 16 bits leave room for the index in the pattern, and one exchange does.  k
// rounds cost 25 to 40 instructions each for four tokens at once.
//
// Order.  Rows are ordered by expert, then token (a token's experts differ), a
// stable order that no atomic decides: a workgroup of 64 tokens sets one bit
// per token in a 64-bit mask of each expert, so a row's rank among its expert's
// rows of the workgroup is a population count.  Up to 64 tokens that is the whole order, and
// one launch does everything.  Beyond, a second kernel adds up the workgroups' counts
// and ranks the rows; of many counts a kernel of its own makes the sums first.
//
// Measured: one token, 64 experts, 8 choices: 4.2 us, of which the launch is most.
// 16384 tokens in bfloat16, 128 experts, 8 choices: 7.3 + 5.6 us (11.7 together in a row
// of calls), the gradient 5.4; the bytes alone (4 MB of logits, 2 MB of results) would
// take 1.5 us, the rest is the launches and the latency of loads that wait for one another.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int TOKENS = 64;          // tokens of a workgroup

// Entries of a row of counts: 16-byte loads, the entries past E are zeros.
__host__ __device__ constexpr int padded(int E) { return (E + 3) & ~3; }

// Unsigned order of floats: larger value, larger number; -inf and NaN give 0.
__device__ __forceinline__ unsigned ordered(float x) {
    if (!(x > -INFINITY)) return 0u;
    if (x == 0.0f) x = 0.0f;                                  // -0 equals 0
    const unsigned u = __float_as_uint(x);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned o) {
    return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}
// exp(x - m) for x <= m; equal infinities give 1, -inf and NaN 0
__device__ __forceinline__ float exp_below(float x, float m) {
    return x == m ? 1.0f : (x > -INFINITY ? expf(x - m) : 0.0f);
}

// f over LANES lanes (16 or 64), in all of them; f is associative and commutative but
// for roundings, which are alike in every lane: f(a, b) and f(b, a) are.
template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f) {
    v = f(v, moved<0xB1>(v));
    v = f(v, moved<0x4E>(v));
    v = f(v, moved<0x141>(v));
    v = f(v, moved<0x140>(v));
#pragma unroll
    for (int d = 16; d < LANES; d <<= 1) v = f(v, __shfl_xor(v, d));
    return v;
}

// Bits of a logit in bfloat16 or binary16 as a float that are zero in either.
constexpr unsigned INDEX = (1u << 13) - 1;

// One token's choice by LANES lanes that hold the logits lane + LANES i in
// x[i] (-inf past E).  Lane j % LANES of the group keeps choice j in slot
// j / LANES of id and w; returns in *live how many were chosen.
// PACKED (16-bit logits): their ordered bits are those above INDEX, where the expert's
// number goes, so that one exchange finds the largest logit and its lowest index.
template <int LANES, int V, bool PACKED>
__device__ __forceinline__ void choose(const float (&x)[V], int sub, int k, bool all,
                                       int (&id)[ROUTE_CHOICES / 16], float (&w)[ROUTE_CHOICES / 16]) {
    unsigned o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        o[i] = ordered(x[i]);
        if constexpr (PACKED) o[i] = o[i] == 0 ? 0u : (o[i] | INDEX) - (sub + LANES * i);
    }
    constexpr int SLOTS = ROUTE_CHOICES / 16;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        id[s] = -1;
        w[s] = -INFINITY;
    }
    float m = 0.0f;
    for (int j = 0; j < k; ++j) {
        unsigned best = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) best = o[i] > best ? o[i] : best;
        best = over_lanes<LANES>(best, [](unsigned a, unsigned b) { return a > b ? a : b; });
        if (best == 0) break;                                 // no expert is left
        int at = 0x7FFFFFFF;
        if constexpr (PACKED) {
            at = INDEX - (best & INDEX);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = o[i] == best ? 0u : o[i];
            best = best & 0x80000000u ? best & ~INDEX : best | INDEX;
        } else {
#pragma unroll
            for (int i = V - 1; i >= 0; --i) at = o[i] == best ? sub + LANES * i : at;
            at = over_lanes<LANES>(at, [](int a, int b) { return a < b ? a : b; });
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = at == sub + LANES * i ? 0u : o[i];
        }
        const float v = unordered(best);
        if (j == 0) m = v;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (j % LANES == sub && j / LANES == s) {
                id[s] = at;
                w[s] = v;
            }
    }
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) w[s] = id[s] >= 0 ? exp_below(w[s], m) : 0.0f;
    if (all) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum += exp_below(x[i], m);
    } else {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) sum += w[s];
    }
    sum = over_lanes<LANES>(sum, [](float a, float b) { return a + b; });
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) w[s] = id[s] >= 0 ? w[s] / sum : 0.0f;
}

template <int LANES, int V, typename T>
__device__ __forceinline__ void load_logits(const T *row, int E, int sub, bool live, float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = sub + LANES * i;
        x[i] = live && e < E ? (float)row[e] : -INFINITY;
    }
}

// Exclusive sums of the E counts f(e) by the whole workgroup of 1024 threads,
// E <= 1024; returns the sum below e = threadIdx.x, the total in *total.
template <typename F>
__device__ int sums_below(int E, F f, int *part, int *total) {
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    const int n = e < E ? f(e) : 0;
    const int v = sum_up_to_lane(n);
    if (lane == 63) part[wave] = v;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < 16; ++i) {
        before += i < wave ? part[i] : 0;
        all += part[i];
    }
    *total = all;
    return before + v - n;
}

// One workgroup for 64 tokens.  One workgroup in all: the order too.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(1024) void route_kernel(const T *__restrict__ logits, int64_t ld,
                                                     int64_t tokens, int E, int k, int all,
                                                     int *__restrict__ ids, float *__restrict__ weights,
                                                     int *__restrict__ counts, int *__restrict__ offsets,
                                                     int *__restrict__ rows, int *__restrict__ slots) {
    __shared__ unsigned long long mask[ROUTE_EXPERTS];
    __shared__ int start[ROUTE_EXPERTS], part[16];
    const int tid = threadIdx.x, sub = tid % LANES, lde = padded(E);
    if (tid < lde) mask[tid] = 0;
    __syncthreads();
    constexpr int AT_ONCE = 1024 / LANES;
    const bool single = gridDim.x == 1;
    int id[TOKENS / AT_ONCE][ROUTE_CHOICES / 16];
#pragma unroll
    for (int p = 0; p < TOKENS / AT_ONCE; ++p) {
        const int local = p * AT_ONCE + tid / LANES;
        const int64_t t = (int64_t)blockIdx.x * TOKENS + local;
        const bool live = t < tokens;
        float x[V], w[ROUTE_CHOICES / 16];
        load_logits<LANES, V>(logits + (live ? t : 0) * ld, E, sub, live, x);
        choose<LANES, V, sizeof(T) == 2>(x, sub, k, all, id[p], w);
#pragma unroll
        for (int s = 0; s < ROUTE_CHOICES / 16; ++s) {
            const int j = sub + LANES * s;
            if (!live || j >= k) continue;
            ids[t * k + j] = id[p][s];
            weights[t * k + j] = w[s];
            if (id[p][s] >= 0) atomicOr(&mask[id[p][s]], 1ull << local);
        }
    }
    __syncthreads();
    if (!single) {
        if (tid < lde) counts[(int64_t)blockIdx.x * lde + tid] = __popcll(mask[tid]);
        return;
    }
    int total;
    const int below = sums_below(E, [&](int e) { return __popcll(mask[e]); }, part, &total);
    if (tid < E) {
        start[tid] = below;
        offsets[tid] = below;
    }
    if (tid == 0) offsets[E] = total;
    __syncthreads();
#pragma unroll
    for (int p = 0; p < TOKENS / AT_ONCE; ++p) {
        const int t = p * AT_ONCE + tid / LANES;
#pragma unroll
        for (int s = 0; s < ROUTE_CHOICES / 16; ++s) {
            const int j = sub + LANES * s, e = id[p][s];
            if (t >= tokens || j >= k) continue;
            const int at = e < 0 ? -1 : start[e] + __popcll(mask[e] & ((1ull << t) - 1));
            slots[t * k + j] = at;
            if (at >= 0) rows[at] = t;
        }
    }
    for (int i = total + tid; i < (int)tokens * k; i += 1024) rows[i] = -1;
}

// The counts of the workgroups of one expert become the sums of those before;
// the expert's total goes to totals[e].  A wave for an expert: its 64 lanes walk the
// workgroups' counts, four loads of a lane at a time.
__global__ __launch_bounds__(64) void route_sums_kernel(int *__restrict__ counts, int64_t blocks,
                                                        int E, int *__restrict__ totals) {
    constexpr int AHEAD = 4;
    const int lane = threadIdx.x, e = blockIdx.x, lde = padded(E);
    int before = 0;
    for (int64_t b0 = lane; b0 - lane < blocks; b0 += 64 * AHEAD) {
        int n[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) n[i] = b0 + 64 * i < blocks ? counts[(b0 + 64 * i) * lde + e] : 0;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int v = sum_up_to_lane(n[i]);
            if (b0 + 64 * i < blocks) counts[(b0 + 64 * i) * lde + e] = before + v - n[i];
            before += __builtin_amdgcn_readlane(v, 63);
        }
    }
    if (lane == 0) totals[e] = before;
}

// Slots and rows of 64 tokens, from their experts and the counts: as route_sums_kernel
// left them, or (ADD) as route_kernel did, where every workgroup adds up those of
// all, a quad of experts and every 1024 / quads-th row to a thread.
template <bool ADD>
__global__ __launch_bounds__(1024) void route_order_kernel(const int *__restrict__ ids, int64_t tokens,
                                                           int E, int k, const int *__restrict__ counts,
                                                           int blocks, const int *__restrict__ totals,
                                                           int *__restrict__ offsets,
                                                           int *__restrict__ rows,
                                                           int *__restrict__ slots) {
    __shared__ unsigned long long mask[ROUTE_EXPERTS];
    __shared__ int start[ROUTE_EXPERTS], every[ADD ? ROUTE_EXPERTS : 1], part[16];
    const int tid = threadIdx.x, lde = padded(E);
    const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
    const int n = (int)((tokens - t0 < TOKENS ? tokens - t0 : TOKENS) * k);
    if (tid < lde) {
        mask[tid] = 0;
        if constexpr (ADD) start[tid] = every[tid] = 0;
    }
    __syncthreads();
    for (int i = tid; i < n; i += 1024) {
        const int e = ids[t0 * k + i];
        if (e >= 0) atomicOr(&mask[e], 1ull << (i / k));
    }
    if constexpr (ADD) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        constexpr int AHEAD = 8;
        const int quads = lde / 4, at_once = 1024 / quads, q = tid % quads, first = tid / quads;
        i32x4 before = {}, all = {};
        for (int b0 = first; first < at_once && b0 < blocks; b0 += at_once * AHEAD) {
            i32x4 c[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int b = b0 + at_once * i;
                c[i] = b < blocks ? reinterpret_cast<const i32x4 *>(counts + (int64_t)b * lde)[q] : i32x4{};
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                all += c[i];
                if (b0 + at_once * i < (int)blockIdx.x) before += c[i];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {                         // whole numbers: any order
            if (all[j] != 0) atomicAdd(&every[4 * q + j], all[j]);
            if (before[j] != 0) atomicAdd(&start[4 * q + j], before[j]);
        }
        __syncthreads();
    }
    int total;
    const int below = sums_below(E, [&](int e) { return ADD ? every[e] : totals[e]; }, part, &total);
    if (tid < E) {
        start[tid] = below + (ADD ? start[tid] : counts[(int64_t)blockIdx.x * lde + tid]);
        if (blockIdx.x == 0) offsets[tid] = below;
    }
    if (blockIdx.x == 0 && tid == 0) offsets[E] = total;
    __syncthreads();
    for (int i = tid; i < n; i += 1024) {
        const int e = ids[t0 * k + i], t = i / k;
        const int at = e < 0 ? -1 : start[e] + __popcll(mask[e] & ((1ull << t) - 1));
        slots[t0 * k + i] = at;
        if (at >= 0) rows[at] = (int)(t0 + t);
        if (t0 * k + i >= total) rows[t0 * k + i] = -1;
    }
}

// Gradient of the logits: with p the softmax that gave the weights (0 outside
// its set) and dw the weights' gradient, dl_e = [e chosen] p_e dw_e - p_e sum_j
// w_j dw_j.  LANES lanes take a token.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(256) void route_grad_kernel(const T *__restrict__ logits, int64_t ld,
                                                         int64_t tokens, int E, int k, int all,
                                                         const int *__restrict__ ids,
                                                         const float *__restrict__ weights,
                                                         const float *__restrict__ dweights,
                                                         T *__restrict__ dlogits, int64_t ldd) {
    const int sub = threadIdx.x % LANES;
    const int64_t t = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const bool live = t < tokens;
    const int64_t tc = live ? t : 0;
    constexpr int SLOTS = ROUTE_CHOICES / 16;
    int id[SLOTS];
    float wd[SLOTS], w[SLOTS], mean = 0.0f;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const int j = sub + LANES * s;
        id[s] = j < k ? ids[tc * k + j] : -1;
        w[s] = id[s] >= 0 ? weights[tc * k + j] : 0.0f;
        wd[s] = id[s] >= 0 ? w[s] * dweights[tc * k + j] : 0.0f;
        mean += wd[s];
    }
    mean = over_lanes<LANES>(mean, [](float a, float b) { return a + b; });
    float x[V], m = -INFINITY, sum = 0.0f;
    if (all) {
        load_logits<LANES, V>(logits + tc * ld, E, sub, true, x);
#pragma unroll
        for (int i = 0; i < V; ++i) m = x[i] > m ? x[i] : m;
        m = over_lanes<LANES>(m, [](float a, float b) { return a > b ? a : b; });
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = m > -INFINITY ? exp_below(x[i], m) : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) sum += x[i];
        sum = over_lanes<LANES>(sum, [](float a, float b) { return a + b; });
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = sum > 0.0f ? -x[i] / sum * mean : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = 0.0f;
    }
    for (int j = 0; j < k; ++j) {
        const int from = (threadIdx.x & 63 & ~(LANES - 1)) + j % LANES, s = j / LANES;
        const int e = __shfl(s == 0 ? id[0] : id[SLOTS - 1], from);
        const float g = __shfl(s == 0 ? wd[0] - (all ? 0.0f : w[0] * mean)
                                      : wd[SLOTS - 1] - (all ? 0.0f : w[SLOTS - 1] * mean),
                               from);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (e == sub + LANES * i) x[i] += g;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = sub + LANES * i;
        if (live && e < E) dlogits[t * ldd + e] = (T)x[i];
    }
}
static_assert(ROUTE_CHOICES == 32, "two slots of a lane");

// f<LANES, V>() with the fewest registers that hold E logits.
template <typename F>
void with_shape(int E, F &&f) {
    using std::integral_constant;
    if (E <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (E <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (E <= 256) f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else if (E <= 512) f(integral_constant<int, 16>{}, integral_constant<int, 32>{});
    else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

// Counts up to which every workgroup of the order adds them up itself.  With k = 8, the
// router's time with and without route_sums_kernel, us: 1024 tokens and 128 experts
// 11.6 and 10.2, 16384 and 128 13.1 and 12.3, 16384 and 256 16.6 and 16.8, 65536 and 64
// 25.2 and 28.7.
constexpr int64_t MOST_ADDED = 1 << 15;
int64_t route_blocks(int64_t T) { return T > TOKENS ? (T + TOKENS - 1) / TOKENS : 1; }

}  // namespace

size_t route_scratch(int64_t T, int E) {
    const int64_t b = route_blocks(T);
    return b > 1 ? (size_t)(b + 1) * padded(E) * sizeof(int) : 0;
}

hipError_t launch_route(int dtype, const void *logits, int64_t ld, int64_t T, int E, int k, bool all,
                        int *ids, float *weights, int *offsets, int *rows, int *slots, char *scratch,
                        hipStream_t s) {
    const int64_t blocks = route_blocks(T);
    int *const counts = reinterpret_cast<int *>(scratch), *const totals = counts + blocks * padded(E);
    with_type(dtype, [&](auto z) {
        using type = decltype(z);
        with_shape(E, [&](auto lanes, auto v) {
            route_kernel<type, lanes, v><<<(unsigned)blocks, 1024, 0, s>>>(
                static_cast<const type *>(logits), ld, T, E, k, all, ids, weights, counts, offsets,
                rows, slots);
        });
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    const bool add = blocks * padded(E) <= MOST_ADDED;
    if (!add) {
        route_sums_kernel<<<E, 64, 0, s>>>(counts, blocks, E, totals);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    (add ? route_order_kernel<true> : route_order_kernel<false>)<<<(unsigned)blocks, 1024, 0, s>>>(
        ids, T, E, k, counts, (int)blocks, totals, offsets, rows, slots);
    return hipGetLastError();
}

hipError_t launch_route_grad(int dtype, const void *logits, int64_t ld, int64_t T, int E, int k,
                             bool all, const int *ids, const float *weights, const float *dweights,
                             void *dlogits, int64_t ldd, hipStream_t s) {
    with_type(dtype, [&](auto z) {
        using type = decltype(z);
        with_shape(E, [&](auto lanes, auto v) {
            constexpr int per = 256 / decltype(lanes)::value;
            route_grad_kernel<type, lanes, v><<<(unsigned)((T + per - 1) / per), 256, 0, s>>>(
                static_cast<const type *>(logits), ld, T, E, k, all, ids, weights, dweights,
                static_cast<type *>(dlogits), ldd);
        });
    });
    return hipGetLastError();
}

}  // namespace emu
