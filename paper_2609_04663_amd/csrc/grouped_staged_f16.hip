#include "grouped_staged.h"

namespace emu {
hipError_t launch_staged_gemm_f16(const GroupedGemm &g, hipStream_t s) { return run_staged_gemm<half>(g, s); }
hipError_t launch_staged_wgrad_f16(const GroupedWgrad &g, hipStream_t s) { return run_staged_wgrad<half>(g, s); }
}  // namespace emu
