// Which kernels run a grouped product.
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int BK = 64;                               // k-block of the kernels of grouped16.h
constexpr int64_t OFFSETS = (int64_t)1 << 32;       // what a copy's 32-bit offset spans

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

// The kernels of grouped16.h: whole 16-byte chunks and k-blocks, and offsets of 32 bits.
static bool direct_gemm(const GroupedGemm &g) {
    return g.dtype != EMU_F32 && g.K >= 2 * BK && g.K % BK == 0 && aligned16(g.X) && aligned16(g.W) &&
           g.ldx % 8 == 0 && g.ldw % 8 == 0 && g.sw % 8 == 0 && (g.transb || g.N % 8 == 0) && g.E > 0 &&
           (g.rows ? g.xrows : 256) * g.ldx * 2 < OFFSETS && 256 * g.ldw * 2 < OFFSETS &&
           (!g.rows || g.xrows > 0);
}
static bool direct_wgrad(const GroupedWgrad &g) {
    return g.dtype != EMU_F32 && aligned16(g.P) && aligned16(g.Q) && g.ldp % 8 == 0 && g.ldq % 8 == 0 &&
           g.M % 8 == 0 && g.N % 8 == 0 && g.ldp * 2 < OFFSETS && g.ldq * 2 < OFFSETS;
}

// Rows per expert up to which the kernel for few rows is the faster one.  Measured, us,
// that kernel and the other one, 64 experts of 2048 x 2048:
//   16 bits, copied straight to LDS   8 rows 112 and 124, 16 rows 119 and 94
//   float32                          32 rows 306 and 615 ('T' 303 to 343 and 433),
//                                    64 rows 600 and 623 ('T' 757 and 436)
//   16 bits, 2041 x 2041 'N'         30 rows 230 and 326, 50 rows 438 and 326
//                        'T'          8 rows 191 and 161
// A rule on the average: where the rows lie is known on the device only.
static int64_t few_rows(const GroupedGemm &g, bool direct) {
    return g.dtype == EMU_F32 || (!direct && !g.transb) ? FEW_ROWS : 8;
}

hipError_t launch_grouped_gemm(const GroupedGemm &g, hipStream_t s) {
    const bool direct = direct_gemm(g), bf16 = g.dtype == EMU_BF16;
    if (g.R <= few_rows(g, direct) * g.E) return launch_few(g, s);
    if (direct) {
        const int tile = g.R >= 512 * (int64_t)g.E ? 256 : 128;
        return bf16 ? launch_gemm16_bf16(g, tile, s) : launch_gemm16_f16(g, tile, s);
    }
    if (g.dtype == EMU_F32) return launch_staged_gemm_f32(g, s);
    return bf16 ? launch_staged_gemm_bf16(g, s) : launch_staged_gemm_f16(g, s);
}

hipError_t launch_grouped_wgrad(const GroupedWgrad &g, hipStream_t s) {
    const bool bf16 = g.dtype == EMU_BF16;
    if (direct_wgrad(g)) {
        const int tile = g.M >= 512 && g.N >= 512 ? 256 : 128;
        return bf16 ? launch_wgrad16_bf16(g, tile, s) : launch_wgrad16_f16(g, tile, s);
    }
    if (g.dtype == EMU_F32) return launch_staged_wgrad_f32(g, s);
    return bf16 ? launch_staged_wgrad_bf16(g, s) : launch_staged_wgrad_f16(g, s);
}

}  // namespace emu
