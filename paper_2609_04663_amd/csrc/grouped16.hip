// When the grouped products of 16-bit operands take the kernels of grouped16.h.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int BK = 64;                               // their k-block
constexpr int64_t OFFSETS = (int64_t)1 << 32;       // what a copy's 32-bit offset spans

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

// Whole 16-byte chunks and k-blocks, and offsets of 32 bits.
bool direct_gemm(const GroupedGemm &g) {
    return g.dtype != EMU_F32 && g.K >= 2 * BK && g.K % BK == 0 && aligned16(g.X) && aligned16(g.W) &&
           g.ldx % 8 == 0 && g.ldw % 8 == 0 && g.sw % 8 == 0 && (g.transb || g.N % 8 == 0) && g.E > 0 &&
           (g.rows ? g.xrows : 256) * g.ldx * 2 < OFFSETS && 256 * g.ldw * 2 < OFFSETS &&
           (!g.rows || g.xrows > 0);
}
bool direct_wgrad(const GroupedWgrad &g) {
    return g.dtype != EMU_F32 && aligned16(g.P) && aligned16(g.Q) && g.ldp % 8 == 0 && g.ldq % 8 == 0 &&
           g.M % 8 == 0 && g.N % 8 == 0 && g.ldp * 2 < OFFSETS && g.ldq * 2 < OFFSETS;
}

hipError_t launch_direct_gemm(const GroupedGemm &g, int tile, hipStream_t s) {
    return g.dtype == EMU_BF16 ? launch_gemm16_bf16(g, tile, s) : launch_gemm16_f16(g, tile, s);
}
hipError_t launch_direct_wgrad(const GroupedWgrad &g, int tile, hipStream_t s) {
    return g.dtype == EMU_BF16 ? launch_wgrad16_bf16(g, tile, s) : launch_wgrad16_f16(g, tile, s);
}

}  // namespace emu
