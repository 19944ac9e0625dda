#include "grouped16.h"

namespace emu {
hipError_t launch_gemm16_f16(const GroupedGemm &g, int tile, hipStream_t s) {
    return launch_gemm16<half>(g, tile, s);
}
}  // namespace emu
