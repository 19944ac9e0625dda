// Packing of matrices into 4 bits, and the choice of the product's source file.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

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

int launch_q4_gemm(const Q4Gemm &g, hipStream_t s) {
    if (g.dtype == EMU_F32) return launch_q4_gemm_f32(g, s);
    if (g.dtype == EMU_BF16) return launch_q4_gemm_bf16(g, s);
    return launch_q4_gemm_f16(g, s);
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
