#include "grouped_staged.h"

namespace emu {
hipError_t launch_staged_gemm_bf16(const GroupedGemm &g, hipStream_t s) { return run_staged_gemm<bhalf>(g, s); }
hipError_t launch_staged_wgrad_bf16(const GroupedWgrad &g, hipStream_t s) { return run_staged_wgrad<bhalf>(g, s); }
}  // namespace emu
