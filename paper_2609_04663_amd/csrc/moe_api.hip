// Entry points of the mixture-of-experts operators declared in include/emu.h:
// argument checks (before any HIP call), degenerate sizes and launches on the
// current stream.
#include <initializer_list>

#include "api_state.h"
#include "moe.h"
#include "moe_common.h"

namespace {

using namespace emu;

constexpr int64_t MAX_TOKENS = (1 << 24) - 1, MAX_ROWS = 0x7FFFFFFF, MAX_COLS = (1 << 30) - 1;
constexpr int64_t MAX_TILES = (1 << 24) - 8;        // workgroups of 256 threads in a launch

int64_t at_least_1(int64_t n) { return n > 1 ? n : 1; }

int check_type(int dtype) {
    return is_dtype(dtype) ? EMU_OK : api_fail(EMU_EINVAL, "dtype must be EMU_F32, EMU_BF16 or EMU_F16");
}

int check_route(int dtype, int64_t T, int E, int k, int scope, int64_t ld) {
    if (int rc = check_type(dtype)) return rc;
    if (T < 0 || T > MAX_TOKENS) return api_fail(EMU_EINVAL, "T out of range");
    if (E < 1 || E > ROUTE_EXPERTS) return api_fail(EMU_EINVAL, "E must be 1 to 1024");
    if (k < 1 || k > E || k > ROUTE_CHOICES) return api_fail(EMU_EINVAL, "k must be 1 to min(E, 32)");
    if (scope != EMU_ROUTE_CHOSEN && scope != EMU_ROUTE_ALL)
        return api_fail(EMU_EINVAL, "scope must be EMU_ROUTE_CHOSEN or EMU_ROUTE_ALL");
    if (ld < E) return api_fail(EMU_EINVAL, "leading dimension < E");
    return EMU_OK;
}

int check_combine(int dtype, int64_t T, int64_t D, int k, int64_t R) {
    if (int rc = check_type(dtype)) return rc;
    if (T < 0 || T > MAX_TOKENS || D < 0 || D > MAX_COLS || R < 0 || R > MAX_ROWS)
        return api_fail(EMU_EINVAL, "T, D or R out of range");
    if (k < 1 || k > ROUTE_CHOICES) return api_fail(EMU_EINVAL, "k must be 1 to 32");
    return EMU_OK;
}

// Leading dimensions of the grouped products: 32-bit multiples in the kernels.
int check_lds(std::initializer_list<int64_t> lds) {
    for (int64_t ld : lds)
        if (ld > MAX_ROWS) return api_fail(EMU_EINVAL, "leading dimension above 2^31 - 1");
    return EMU_OK;
}

// Sizes and index arrays that the grouped products share.
int check_grouped(int dtype, int E, int64_t R, int64_t N, int64_t K, int64_t XR, const void *rows,
                  const void *offsets, bool need_offsets) {
    if (int rc = check_type(dtype)) return rc;
    if (E < 0 || E > 1 << 16) return api_fail(EMU_EINVAL, "E must be 0 to 65536");
    if (R < 0 || R > MAX_ROWS || XR < 0 || XR > MAX_ROWS) return api_fail(EMU_EINVAL, "R or XR out of range");
    if (N < 0 || N > MAX_COLS || K < 0 || K > MAX_COLS) return api_fail(EMU_EINVAL, "N or K out of range");
    if (!rows && XR < R) return api_fail(EMU_EINVAL, "X has fewer than R rows and rows is NULL");
    if (need_offsets && !offsets) return api_fail(EMU_EINVAL, "offsets is NULL");
    return EMU_OK;
}

int trans(char t, bool *tr) {
    if (t == 'N' || t == 'n') *tr = false;
    else if (t == 'T' || t == 't') *tr = true;
    else return api_fail(EMU_EINVAL, "transb must be 'N' or 'T'");
    return EMU_OK;
}

}  // namespace

extern "C" {

int emu_moe_route(int dtype, int64_t T, int E, int k, int scope, const void *logits, int64_t ldl,
                  int32_t *ids, float *weights, int32_t *offsets, int32_t *rows, int32_t *slots) {
    if (int rc = check_route(dtype, T, E, k, scope, ldl)) return rc;
    if (!offsets) return api_fail(EMU_EINVAL, "offsets is NULL");
    if (T > 0 && (!logits || !ids || !weights || !rows || !slots))
        return api_fail(EMU_EINVAL, "NULL pointer");
    api_clear_error();
    char *scratch = nullptr;
    const size_t need = route_scratch(T, E);
    if (need > 0)
        if (int rc = api_workspace(need, &scratch)) return rc;
    // T = 0: one workgroup without tokens writes the offsets
    return api_done(launch_route(dtype, logits, ldl, T, E, k, scope == EMU_ROUTE_ALL, ids, weights, offsets,
                                 rows, slots, scratch, api_stream()), "moe_route");
}

int emu_moe_route_grad(int dtype, int64_t T, int E, int k, int scope, const void *logits, int64_t ldl,
                       const int32_t *ids, const float *weights, const float *dweights,
                       void *dlogits, int64_t ldd) {
    if (int rc = check_route(dtype, T, E, k, scope, ldd)) return rc;
    if (scope == EMU_ROUTE_ALL && ldl < E) return api_fail(EMU_EINVAL, "leading dimension < E");
    if (T > 0 && ((scope == EMU_ROUTE_ALL && !logits) || !ids || !weights || !dweights || !dlogits))
        return api_fail(EMU_EINVAL, "NULL pointer");
    api_clear_error();
    if (T == 0) return EMU_OK;
    return api_done(launch_route_grad(dtype, logits, ldl, T, E, k, scope == EMU_ROUTE_ALL, ids, weights,
                                      dweights, dlogits, ldd, api_stream()), "moe_route_grad");
}

int emu_moe_combine(int dtype, int64_t T, int64_t D, int k, int64_t R, const void *Z, int64_t ldz,
                    const int32_t *slots, const float *weights, void *Y, int64_t ldy) {
    if (int rc = check_combine(dtype, T, D, k, R)) return rc;
    if (ldz < at_least_1(D) || ldy < at_least_1(D)) return api_fail(EMU_EINVAL, "leading dimension < max(1, D)");
    if (T > 0 && D > 0 && ((R > 0 && !Z) || !slots || !Y)) return api_fail(EMU_EINVAL, "NULL pointer");
    api_clear_error();
    if (T == 0 || D == 0) return EMU_OK;
    return api_done(launch_combine(dtype, Z, ldz, R, T, D, k, slots, weights, Y, ldy, api_stream()),
                    "moe_combine");
}

int emu_moe_combine_grad(int dtype, int64_t T, int64_t D, int k, int64_t R, const void *dY,
                         int64_t lddy, const void *Z, int64_t ldz, const int32_t *slots,
                         const float *weights, const int32_t *rows, void *dZ, int64_t lddz,
                         float *dweights) {
    if (int rc = check_combine(dtype, T, D, k, R)) return rc;
    if (lddy < at_least_1(D) || ldz < at_least_1(D) || lddz < at_least_1(D))
        return api_fail(EMU_EINVAL, "leading dimension < max(1, D)");
    if (T > 0 && ((D > 0 && (!dY || (R > 0 && !Z))) || !slots || !weights || !dweights))
        return api_fail(EMU_EINVAL, "NULL pointer");
    if (R > 0 && (!rows || (D > 0 && !dZ))) return api_fail(EMU_EINVAL, "NULL pointer");
    api_clear_error();
    if (T == 0 && (R == 0 || D == 0)) return EMU_OK;
    return api_done(launch_combine_grad(dtype, dY, lddy, Z, ldz, R, T, D, k, slots, weights, rows, dZ, lddz,
                                        dweights, api_stream()), "moe_combine_grad");
}

int emu_grouped_gemm(int dtype, char transb, int E, int64_t R, int64_t N, int64_t K, const void *X,
                     int64_t ldx, int64_t XR, const int32_t *rows, const void *W, int64_t ldw,
                     int64_t stride, const int32_t *offsets, void *Y, int64_t ldy) {
    bool tb = false;
    if (int rc = trans(transb, &tb)) return rc;
    if (int rc = check_grouped(dtype, E, R, N, K, XR, rows, offsets, R > 0 && N > 0)) return rc;
    if (ldx < at_least_1(K) || ldw < at_least_1(tb ? K : N) || ldy < at_least_1(N))
        return api_fail(EMU_EINVAL, "leading dimension below the row length");
    if (stride < 0) return api_fail(EMU_EINVAL, "stride < 0");
    if (R > 0 && N > 0 && (!Y || (K > 0 && E > 0 && ((XR > 0 && !X) || !W))))
        return api_fail(EMU_EINVAL, "NULL pointer");
    if (int rc = check_lds({ldx, ldw, ldy})) return rc;
    // workgroups of 512 threads: on tiles of 16 x 64 or more where the rows are few, else of 128 x 128
    const int64_t tiles = R <= FEW_ROWS * E ? row_blocks_bound(R, E, 16) * ((N + 63) / 64)
                                            : row_blocks_bound(R, E, 128) * ((N + 127) / 128);
    if (tiles > MAX_TILES / 2) return api_fail(EMU_EINVAL, "product too large");
    api_clear_error();
    if (R == 0 || N == 0) return EMU_OK;
    const GroupedGemm g = {dtype, E, (int)N, (int)K, R, XR, X, W, Y, ldx, ldw, stride, ldy, offsets, rows, tb};
    return launch_grouped_gemm(g, api_stream());
}

int emu_grouped_wgrad(int dtype, char transb, int E, int64_t R, int64_t N, int64_t K, const void *X,
                      int64_t ldx, int64_t XR, const int32_t *rows, const void *dY, int64_t lddy,
                      const int32_t *offsets, void *dW, int64_t ldw, int64_t stride) {
    bool tb = false;
    if (int rc = trans(transb, &tb)) return rc;
    if (int rc = check_grouped(dtype, E, R, N, K, XR, rows, offsets, E > 0 && N > 0 && K > 0)) return rc;
    if (ldx < at_least_1(K) || lddy < at_least_1(N) || ldw < at_least_1(tb ? K : N))
        return api_fail(EMU_EINVAL, "leading dimension below the row length");
    if (stride < 0) return api_fail(EMU_EINVAL, "stride < 0");
    if (E > 0 && N > 0 && K > 0 && (!dW || (R > 0 && ((XR > 0 && !X) || !dY))))
        return api_fail(EMU_EINVAL, "NULL pointer");
    if (int rc = check_lds({ldx, lddy, ldw})) return rc;
    if (E > 1 && N > 0 && K > 0 && stride < ((tb ? N : K) - 1) * ldw + (tb ? K : N))
        return api_fail(EMU_EINVAL, "the matrices of dW overlap");
    if (E * ((N + 127) / 128) * ((K + 127) / 128) > MAX_TILES / 2) return api_fail(EMU_EINVAL, "product too large");
    api_clear_error();
    if (E == 0 || N == 0 || K == 0) return EMU_OK;
    // dW as stored: X^T dY (K x N), or its transpose dY^T X
    const GroupedWgrad g = tb ? GroupedWgrad{dtype, E, (int)N, (int)K, R, R, XR, dY, X, dW, lddy, ldx,
                                             ldw, stride, offsets, nullptr, rows, 1}
                              : GroupedWgrad{dtype, E, (int)K, (int)N, R, XR, R, X, dY, dW, ldx, lddy,
                                             ldw, stride, offsets, rows, nullptr, 1};
    return launch_grouped_wgrad(g, api_stream());
}

int emu_q4_gemm(int dtype, int E, int64_t R, int64_t N, int64_t K, int group, const void *X,
                int64_t ldx, int64_t XR, const int32_t *rows, const uint8_t *Q, const void *scales,
                const void *mins, const int32_t *offsets, void *Y, int64_t ldy) {
    if (group != 32 && group != 64 && group != 128) return api_fail(EMU_EINVAL, "group must be 32, 64 or 128");
    if (int rc = check_grouped(dtype, E, R, N, K, XR, rows, offsets, R > 0 && N > 0 && E != 1)) return rc;
    if (K % group != 0) return api_fail(EMU_EINVAL, "K must be a multiple of the group");
    if (ldx < at_least_1(K) || ldy < at_least_1(N))
        return api_fail(EMU_EINVAL, "leading dimension below the row length");
    if (R > 0 && N > 0 && (!Y || (K > 0 && E > 0 && ((XR > 0 && !X) || !Q || !scales))))
        return api_fail(EMU_EINVAL, "NULL pointer");
    // workgroups of 512 threads: where they are many, a column of 128 or more at a time and sixteen
    // of these one after the other
    if (R > 0 && row_blocks_bound(R, E, q4_tile_rows(dtype, R, at_least_1(E))) * ((N + 2047) / 2048) > MAX_TILES / 2)
        return api_fail(EMU_EINVAL, "product too large");
    api_clear_error();
    if (R == 0 || N == 0) return EMU_OK;
    const Q4Gemm g = {dtype, E, (int)N, (int)K, group, R, XR, X, Q, scales, mins, Y, ldx, ldy, offsets, rows};
    return launch_q4_gemm(g, api_stream());
}

int emu_q4_pack(int dtype, int64_t rows, int64_t K, int group, const void *W, int64_t ldw, uint8_t *Q,
                void *scales) {
    if (int rc = check_type(dtype)) return rc;
    if (group != 32 && group != 64 && group != 128) return api_fail(EMU_EINVAL, "group must be 32, 64 or 128");
    if (rows < 0 || rows > MAX_ROWS || K < 0 || K > MAX_COLS) return api_fail(EMU_EINVAL, "rows or K out of range");
    if (K % group != 0) return api_fail(EMU_EINVAL, "K must be a multiple of the group");
    if (ldw < at_least_1(K)) return api_fail(EMU_EINVAL, "ldw < max(1, K)");
    if (rows > 0 && K > 0 && (!W || !Q || !scales)) return api_fail(EMU_EINVAL, "NULL pointer");
    if (K > 0 && rows > (((int64_t)1 << 32) - 256) / (K / 8)) return api_fail(EMU_EINVAL, "matrix too large");
    api_clear_error();
    if (rows == 0 || K == 0) return EMU_OK;
    return api_done(launch_q4_pack(dtype, W, rows, ldw, (int)K, group, Q, scales, api_stream()), "q4_pack");
}

}  // extern "C"
