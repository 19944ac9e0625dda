#include "grouped_staged.h"

namespace emu {
hipError_t launch_staged_gemm_f32(const GroupedGemm &g, hipStream_t s) { return run_staged_gemm<float>(g, s); }
hipError_t launch_staged_wgrad_f32(const GroupedWgrad &g, hipStream_t s) { return run_staged_wgrad<float>(g, s); }
}  // namespace emu
