#include "q8_tiles.h"

namespace emu {
hipError_t launch_q8_tiles_f16(const Q8Gemm &g, Q8Tiles how, hipStream_t s) {
    return launch_q8_tiles<half>(g, how, s);
}
}  // namespace emu
