// Launch wrappers of the mixture-of-experts kernels (arguments checked by the
// entry points in moe_api.hip).  Those that may ask for workspace return an EMU_*
// code and set its message, the others HIP's.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace emu {

constexpr int ROUTE_EXPERTS = 1024, ROUTE_CHOICES = 32;   // most experts, most choices of a token

// Bytes of scratch that a routing of T tokens over E experts needs.
size_t route_scratch(int64_t T, int E);
hipError_t launch_route(int dtype, const void *logits, int64_t ld, int64_t T, int E, int k, bool all,
                        int *ids, float *weights, int *offsets, int *rows, int *slots, char *scratch,
                        hipStream_t s);
hipError_t launch_route_grad(int dtype, const void *logits, int64_t ld, int64_t T, int E, int k,
                             bool all, const int *ids, const float *weights, const float *dweights,
                             void *dlogits, int64_t ldd, hipStream_t s);
hipError_t launch_combine(int dtype, const void *Z, int64_t ldz, int64_t R, int64_t T, int64_t D,
                          int k, const int *slots, const float *weights, void *Y, int64_t ldy,
                          hipStream_t s);
hipError_t launch_combine_grad(int dtype, const void *dY, int64_t lddy, const void *Z, int64_t ldz,
                               int64_t R, int64_t T, int64_t D, int k, const int *slots,
                               const float *weights, const int *rows, void *dZ, int64_t lddz,
                               float *dweights, hipStream_t s);

// The balance loss and its gradient; see emu_moe_balance.
struct BalanceLoss {
    int dtype, E, k, S;
    int64_t T, ld;
    const void *logits;
    const int *ids, *starts;
    float *loss, *zloss;
    int *counts, *tokens;
};
struct BalanceGrad {
    int dtype, E, S;
    int64_t T, ld, ldd;
    const void *logits;
    const int *counts, *tokens, *starts;
    const float *dloss, *dzloss;
    void *dlogits;
};
// Bytes of scratch that the loss of T tokens in S sequences needs.
size_t balance_scratch(int64_t T, int E, int S);
hipError_t launch_balance(const BalanceLoss &b, char *scratch, hipStream_t s);
hipError_t launch_balance_grad(const BalanceGrad &b, hipStream_t s);

// Products of rows ordered by expert; see emu_grouped_gemm and emu_grouped_wgrad.
struct GroupedGemm {
    int dtype, E, N, K;
    int64_t R, xrows;               // rows of the product; rows of X
    const void *X, *W;
    void *Y;
    int64_t ldx, ldw, sw, ldy;
    const int *offsets, *rows;
    bool transb;
};
int launch_grouped_gemm(const GroupedGemm &g, hipStream_t s);
struct GroupedWgrad {
    int dtype, E, M, N;             // dW[e] is M x N = sum over its rows of P[r]^T Q[r]
    int64_t R, prows, qrows;
    const void *P, *Q;
    void *dW;
    int64_t ldp, ldq, ldw, sw;
    const int *offsets, *prow, *qrow;   // row numbers of P and Q, or null: r itself
    // An expert's rows in this many pieces, each with its own sum: FP32 matrices
    // dW[e pieces + i], ldw a multiple of 4, sw entries apart.
    int pieces;
};
int launch_grouped_wgrad(const GroupedWgrad &g, hipStream_t s);

// The kernels of 16-bit operands copied straight to LDS (grouped16.h), with square
// output tiles of 128 or 256; one source file each: they take long to compile.
hipError_t launch_gemm16_bf16(const GroupedGemm &g, int tile, hipStream_t s);
hipError_t launch_gemm16_f16(const GroupedGemm &g, int tile, hipStream_t s);
hipError_t launch_wgrad16_bf16(const GroupedWgrad &g, int tile, hipStream_t s);
hipError_t launch_wgrad16_f16(const GroupedWgrad &g, int tile, hipStream_t s);
// The kernels staged through registers (grouped_staged.h).
hipError_t launch_staged_gemm_f32(const GroupedGemm &g, hipStream_t s);
hipError_t launch_staged_gemm_bf16(const GroupedGemm &g, hipStream_t s);
hipError_t launch_staged_gemm_f16(const GroupedGemm &g, hipStream_t s);
hipError_t launch_staged_wgrad_f32(const GroupedWgrad &g, hipStream_t s);
hipError_t launch_staged_wgrad_bf16(const GroupedWgrad &g, hipStream_t s);
hipError_t launch_staged_wgrad_f16(const GroupedWgrad &g, hipStream_t s);
// The kernel for a few rows of each expert: at most FEW_ROWS of each on average.
constexpr int64_t FEW_ROWS = 32;
hipError_t launch_few(const GroupedGemm &g, hipStream_t s);

// Products with 4-bit matrices; see emu_q4_gemm and emu_q4_pack.
struct Q4Gemm {
    int dtype, E, N, K, group;
    int64_t R, xrows;
    const void *X;
    const uint8_t *Q;
    const void *scales, *mins;
    void *Y;
    int64_t ldx, ldy;
    const int *offsets, *rows;
};
int launch_q4_gemm(const Q4Gemm &g, hipStream_t s);
int launch_q4_gemm_f32(const Q4Gemm &g, hipStream_t s);
int launch_q4_gemm_bf16(const Q4Gemm &g, hipStream_t s);
int launch_q4_gemm_f16(const Q4Gemm &g, hipStream_t s);
// Rows of a tile: above 48 of an expert on average 64, for float32 32 (see q4.h).
inline int q4_tile_rows(int dtype, int64_t R, int64_t E) {
    const int64_t sets = (R + 16 * E - 1) / (16 * E);
    return sets <= 3 ? (int)(16 * sets) : (dtype == 0 ? 32 : 64);
}
hipError_t launch_q4_pack(int dtype, const void *W, int64_t rows, int64_t ldw, int K, int group,
                          uint8_t *Q, void *scales, hipStream_t s);

// Rows in 8-bit integers and products of such rows; see emu_q8_pack, emu_q8_unpack and emu_q8_gemm.
hipError_t launch_q8_pack(int dtype, const void *X, int64_t rows, int64_t ldx, int64_t K, int8_t *Q, int64_t ldq,
                          float *scales, hipStream_t s);
hipError_t launch_q8_unpack(int dtype, const int8_t *Q, int64_t rows, int64_t ldq, int64_t K, const float *scales,
                            void *X, int64_t ldx, hipStream_t s);
struct Q8Gemm {
    int dtype, E, N, K;             // dtype: of Y
    int64_t R, xrows;
    const int8_t *X, *W;
    const float *xs, *ws;           // a scale for each row of X; for each row of W, E x N
    void *Y;
    int64_t ldx, ldw, sw, ldy;
    const int *offsets, *rows;
    const int *scaled;              // rows of X that the rows of Y have their scales from: `rows`, also where X is in order
    // Sums: split i of the launch (blockIdx.y) takes the indices i part .. (i + 1) part - 1 and
    // writes its 32-bit sums, without scales, to Y + i R ldy.
    int part;
};
int launch_q8_gemm(const Q8Gemm &g, hipStream_t s);
hipError_t launch_q8_few(const Q8Gemm &g, hipStream_t s);
hipError_t launch_q8_few_sums(const Q8Gemm &g, int splits, hipStream_t s);
// What its time goes by (E > 0): its tiles, their rows and columns in sixteens, how many of
// them share a CU, whether all rows are whole 32-bit words; indices that a workgroup takes at
// a time.
struct Q8FewShape {
    double tiles;
    int mt, nt, per_cu;
    bool words;
};
Q8FewShape q8_few_shape(const Q8Gemm &g);
constexpr int Q8_FEW_ROUND = 1024;
// The kernel of operands copied straight to LDS (q8_tiles.h), with square output tiles of 256,
// or of 128, two workgroups of two stages on a CU or one of four; one source file for each
// type of Y: they take long to compile.
enum class Q8Tiles { LARGE, SMALL, DEEP };
hipError_t launch_q8_tiles_f32(const Q8Gemm &g, Q8Tiles how, hipStream_t s);
hipError_t launch_q8_tiles_bf16(const Q8Gemm &g, Q8Tiles how, hipStream_t s);
hipError_t launch_q8_tiles_f16(const Q8Gemm &g, Q8Tiles how, hipStream_t s);
hipError_t launch_q8_tiles_sums(const Q8Gemm &g, int splits, hipStream_t s);    // DEEP

}  // namespace emu
