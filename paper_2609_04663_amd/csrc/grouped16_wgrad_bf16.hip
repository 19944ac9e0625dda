#include "grouped16.h"

namespace emu {
hipError_t launch_wgrad16_bf16(const GroupedWgrad &g, int tile, hipStream_t s) {
    return launch_wgrad16<bhalf>(g, tile, s);
}
}  // namespace emu
