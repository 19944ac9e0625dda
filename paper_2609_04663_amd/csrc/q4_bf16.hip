#include "q4.h"

namespace emu {
int launch_q4_gemm_bf16(const Q4Gemm &g, hipStream_t s) {
    return run_q4_gemm<bhalf>(g, s);
}
}  // namespace emu
