#include "q8_tiles.h"

namespace emu {
hipError_t launch_q8_tiles_sums(const Q8Gemm &g, int splits, hipStream_t s) {
    const int64_t tiles = row_blocks_bound(g.R, g.E, 128) * ((g.N + 127) / 128);
    const dim3 grid(workgroups(tiles, 1), splits);
    if (g.rows) q8_tiles_kernel<int, 2, 4, true><<<grid, 256, 0, s>>>(g);
    else q8_tiles_kernel<int, 2, 4, false><<<grid, 256, 0, s>>>(g);
    return hipGetLastError();
}
}  // namespace emu
