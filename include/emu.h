/*
 * emu.h -- C ABI of the MI355X (gfx950) library for FP32 and FP64 GEMM
 * emulated through BF16 component products (arxiv 2609.04663).
 *
 * Problem (Sec. 3.2, Eq. gemm): C = A B with A (M x K), B (K x N), C (M x N),
 * all row-major with leading dimensions lda, ldb, ldc counted in elements.
 * emu_sgemm / emu_dgemm have no alpha/beta and no transpose: C is fully
 * overwritten.  The BLAS forms emu_sgemm_ex / emu_dgemm_ex (below) add
 * op(A), op(B) and C = alpha op(A) op(B) + beta C.
 *
 * Pointers.  A, B and C are device pointers (HIP global memory) owned by the
 * caller; A and B are only read.  C must not alias A or B.  Every call is
 * ordered on the library's current stream (emu_set_stream) and returns
 * without synchronising the host; results are ready when that stream is.
 *
 * Workspace.  The library keeps one device workspace per process (packed BF16
 * component planes, per-level exponents, a status word).  It is grown with
 * hipMalloc when a call needs more than it holds -- never on a call whose
 * sizes fit -- and freed by emu_release_workspace.  The environment variable
 * EMU_WORKSPACE_LIMIT (bytes) caps its size; a call that would exceed the cap
 * returns EMU_ENOMEM.
 *
 * Return codes.  EMU_OK on success.  EMU_EINVAL for a bad argument (checked
 * before any HIP call, nothing is launched): M, N or K negative; lda < K,
 * ldb < N, ldc < N (each at least 1); a NULL pointer for an operand with a
 * nonzero extent; nprod not one of the N_p(d) listed at emu_dgemm.  EMU_EHIP
 * when a HIP runtime call or kernel launch fails (message in emu_last_error).
 * EMU_ENOMEM when the workspace cannot be allocated.
 *
 * Degenerate sizes.  M == 0 or N == 0: nothing is done.  K == 0: C = 0.
 *
 * Input domain.  FP32 inputs: any finite value; the three-component split is
 * exact for 2^-103 <= |a| < (2 - 2^-8) 2^127 (Sec. 4.2).  FP64 inputs: the
 * BF16-range domain of Eq. (bf16rangefp64) -- 0 or 2^-126 <= |x| <=
 * (2 - 2^-7) 2^127 -- with every extracted slice a normal BF16 value
 * (Sec. 3.1, 4.3).  As in the paper there is no fallback: out-of-domain input
 * is computed anyway and reported through emu_domain_status; the call itself
 * does not fail.
 *
 * Not thread-safe: one host thread at a time may call into the library.
 */
#ifndef EMU_H
#define EMU_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EMU_OK 0
#define EMU_EINVAL 1
#define EMU_EHIP 2
#define EMU_ENOMEM 3

/* Status bits reported by emu_domain_status. */
#define EMU_STATUS_NAN 1u       /* NaN or infinity in an operand */
#define EMU_STATUS_RANGE 2u     /* finite FP64 input outside Eq. (bf16rangefp64) */
#define EMU_STATUS_SUBNORMAL 4u /* a nonzero component is subnormal in BF16 or
                                   underflowed (the split is not exact) */
#define EMU_STATUS_OVERFLOW 8u  /* a component overflowed BF16 */
#define EMU_STATUS_INEXACT 16u  /* (emu_dgemm) a retained panel product may leave
                                   FP32's exact range: for some (i, j) of the
                                   product set, 2^(vA_i + vB_j - 16) (the unit of
                                   the panel sum) is below 2^-126 or
                                   2^(vA_i + vB_j + 8) (its bound) above 2^127,
                                   so that product may be rounded or overflow in
                                   FP32 and the result is not Eq.
                                   (fp64reconstruction) with exact panel products */

#define EMU_STATUS_FALLBACK 32u /* (emu_dgemm with EMU_FALLBACK_FP64) the call's
                                   split raised a bit above and C was computed by
                                   the native FP64 fallback instead */

/* FP64 split projection constant (Eq. fp64split).  SYM (default) uses
   Sigma = 0.75 * 2^(v+45): granularity 2^(v-8) for both signs, which is the
   reading that reproduces the paper's accuracy table.  LITERAL uses
   Sigma = 2^(v+45) exactly as printed. */
#define EMU_SPLIT_SYM 0
#define EMU_SPLIT_LITERAL 1

/* Exponent scope of the FP64 split (emu_set_split_scope).
   OPERAND (default): the paper's split, one exponent chain v^(r) per operand
   (Eq. fp64split, maxima over the whole operand).
   ROWCOL: the scale-aware form the paper names as its key future step
   (Sec. 9), with stored power-of-two weights as in Eq. (ozakiscaled) at row /
   column granularity: every row m of A is divided by 2^sA_m and every column
   n of B by 2^sB_n, s = ceil(log2 max|x|) over that row or column (0 if it has
   no nonzero finite entry); the scaled operands get the operand-wide split;
   the GEMM multiplies the weights back, C_mn = 2^(sA_m + sB_n) C'_mn.  The
   scalings are exact (powers of two), so the domain becomes: finite inputs
   whose nonzero entries lie within 2^-126 of their row's (A) or column's (B)
   largest magnitude, and results that neither overflow nor underflow FP64. */
#define EMU_SCOPE_OPERAND 0
#define EMU_SCOPE_ROWCOL 1
/* KBIN: the scale-aware form extended along the reduction, for products whose
   terms differ in magnitude along k (for example some rows of B far larger
   than the others), which row and column weights cannot normalise.  With the
   ROWCOL weights sA, sB, the class of reduction index k is
     min(7, floor(-(ceil(log2 max_m |A_mk 2^-sA_m|) + ceil(log2 max_n |B_kn 2^-sB_n|)) / 8))
   (op(A), op(B); an index whose column of op(A) or row of op(B) is zero adds
   exact zeros and is left out).  The indices of each class form a group; each
   group is an emulated DGEMM of its columns of op(A) and rows of op(B) in the
   ROWCOL scope (its own weights and exponent chains), and the groups are added
   in FP64 in ascending class order, S = P_0, then S = fl(P_c + S); the
   call returns fl(fl(alpha S) + fl(beta C)).  The call synchronises its stream
   once (to size the groups) and uses workspace for the gathered groups
   (8 (M + N) K bytes) and, unless alpha = 1 and beta = 0, for S (8 M N).
   Not available to emu_dgemm_noalloc (EMU_EINVAL).  emu_split_f64 and the
   status checks behave as in ROWCOL. */
#define EMU_SCOPE_KBIN 2

/* Emulated SGEMM, Algorithm fp32 (Sec. 4.2, Eq. fp32split and fp32six):
   each FP32 operand is split into three BF16 components; the six products
   A_iB_j with i + j < 3 are evaluated with FP32 accumulation on bf16 MFMA.
   The leading product A0B0 is accumulated per reduction panel of 256 and each
   panel sum is added into an FP32 total; the five smaller products share a
   second FP32 accumulator over the whole reduction (or over each part of a
   split reduction), added to the total at the end.  A: M x K (lda), B: K x N
   (ldb), C: M x N (ldc), device pointers, FP32. */
int emu_sgemm(int64_t M, int64_t N, int64_t K, const float *A, int64_t lda, const float *B,
              int64_t ldb, float *C, int64_t ldc);

/* Emulated DGEMM, Algorithm fp64 (Sec. 4.3, Eq. fp64split, fp64productcounts,
   fp64reconstruction): each FP64 operand gets the fixed six-slice Ozaki split
   with operand-wide exponents; the nprod products A_i B_j with i, j < 6 and
   i + j < d (Eq. product-selection) are each formed in FP32 per reduction
   panel of 256 (exactly, see below), widened and added in FP64 in the order:
   panel ascending, diagonal i + j ascending, i ascending.  nprod = N_p(d):
   6, 10, 15, 21 for the paper's d = 3, 4, 5, 6 (Eq. fp64productcounts), and
   the rest of the selection sequence, 1, 3 (d = 1, 2) and 26, 30, 33, 35, 36
   (d = 7 .. 11; 36 keeps all six-by-six products, Sec. 4.3).
   A: M x K (lda), B: K x N (ldb), C: M x N (ldc), device pointers, FP64.
   For in-domain inputs every panel product is an exact FP32 value, so the
   result is independent of the order of the bf16 MFMA accumulation inside a
   panel. */
int emu_dgemm(int64_t M, int64_t N, int64_t K, const double *A, int64_t lda, const double *B,
              int64_t ldb, double *C, int64_t ldc, int nprod);

/* emu_dgemm for callers that cannot allocate device memory: code under HIP
   graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
   arguments, result and status reporting as emu_dgemm (current stream,
   current split mode and scope), but it never allocates: instead of the
   growing workspace it uses a fixed 64 MiB device array that the library
   holds on every GPU it runs on until the process ends (its address is looked
   up on the first call on each device, which also clears its status word with
   a kernel).  A call whose packed planes (2 min(d, 6) bytes per element of
   both operands; rows padded to whole tiles and two tiles more, K to whole
   k-blocks of 32, or for K > 1024 at d = 3 .. 6 with at least as many output
   tiles as CUs to whole panels of 256) plus a 2 KB header and, in the ROWCOL scope, 12 bytes per row of A and column of B
   exceed 64 MiB returns EMU_ENOMEM before launching anything (square
   problems up to about M = N = K = 1500 at nprod = 21, 2100 at nprod = 6).  All calls on one GPU
   share that array: calls that overlap in time on one GPU (two streams, two
   host threads) race and must be ordered by the caller.  C, A and B are the
   caller's, as for emu_dgemm. */
int emu_dgemm_noalloc(int64_t M, int64_t N, int64_t K, const double *A, int64_t lda,
                      const double *B, int64_t ldb, double *C, int64_t ldc, int nprod);

/* BLAS forms (the "more complete BLAS semantics" of Sec. 9):
     C = alpha op(A) op(B) + beta C,  row-major, op(X) = X or X^T.
   transa, transb: 'N' (op(X) = X) or 'T' ('C' is accepted as 'T'; lower case
   too).  op(A) is M x K: A is M x K with lda >= max(1, K) for 'N', K x M with
   lda >= max(1, M) for 'T'.  op(B) is K x N: B is K x N with ldb >= max(1, N)
   for 'N', N x K with ldb >= max(1, K) for 'T'.  With P the emulated product
   (the value emu_sgemm / emu_dgemm give for op(A) op(B)), each entry becomes
   fl(alpha P) if beta == 0 -- C is then not read and may hold anything -- and
   fl(fl(alpha P) + fl(beta C)) otherwise (no fused multiply-add), so
   alpha = 1, beta = 0 is emu_sgemm / emu_dgemm exactly.  alpha == 0 or K == 0:
   A and B are not read and C = beta C (0 when beta == 0).  Transposed operands
   are packed from their stored layout directly, so op(A) op(B) gives the same
   bits as the plain call on explicitly transposed copies.  Errors as for
   emu_sgemm / emu_dgemm, plus EMU_EINVAL for another transa / transb. */
int emu_sgemm_ex(char transa, char transb, int64_t M, int64_t N, int64_t K, float alpha,
                 const float *A, int64_t lda, const float *B, int64_t ldb, float beta, float *C,
                 int64_t ldc);
int emu_dgemm_ex(char transa, char transb, int64_t M, int64_t N, int64_t K, double alpha,
                 const double *A, int64_t lda, const double *B, int64_t ldb, double beta,
                 double *C, int64_t ldc, int nprod);

/* Fallback of the emulated DGEMM for inputs its split cannot represent (the
   "fallback handling" of Sec. 9 and the "fallback extension" of Sec. 4.3),
   for subsequent emu_dgemm, emu_dgemm_ex and emu_dgemm_noalloc calls.
   EMU_FALLBACK_NONE (default): as in the paper, out-of-domain input is
   computed anyway and only reported.  EMU_FALLBACK_FP64: when the split of
   the call raises any EMU_STATUS_* bit (NaN or infinity, an entry outside
   Eq. (bf16rangefp64) in the current scope, a subnormal, underflowed or
   overflowed slice, a panel product that may be inexact in FP32), C is
   recomputed as alpha op(A) op(B) + beta C by a plain FP64 GEMM (fused
   multiply-adds, its own summation order) and EMU_STATUS_FALLBACK is reported
   as well.  The decision is taken on the device, before the product GEMM, which
   is then left out: no host synchronisation; the armed mode costs a kernel
   launch per call that does nothing unless the fallback is needed.
   EMU_EINVAL for any other value. */
#define EMU_FALLBACK_NONE 0
#define EMU_FALLBACK_FP64 1
int emu_set_fallback(int mode);

/* How subsequent emu_sgemm and emu_sgemm_ex calls split their operands
   (Eq. fp32split; Sec. 6.2 weighs the two ways):
   EMU_SGEMM_SPLIT_PASS (default): a split kernel writes the three BF16 planes
   of both operands to the workspace, and the product kernel reads them;
   EMU_SGEMM_SPLIT_STREAMED: the product kernel reads op(A) and op(B) in FP32
   and splits every k-block itself, in each workgroup that uses it, with the
   split kernel's arithmetic (128 x 128 output tiles): no planes in HBM,
   workspace only for split-reduction partial sums, the same status bits, and
   the same result bits whenever both ways cut the reduction into the same
   number of parts.  EMU_EINVAL for any other value. */
#define EMU_SGEMM_SPLIT_PASS 0
#define EMU_SGEMM_SPLIT_STREAMED 1
int emu_set_sgemm_split(int mode);

/* ---------------------------------------------------------------------------
   Operators of a mixture-of-experts layer: the router and its balance loss, the products with
   the experts' matrices (forward and gradients), with 4-bit expert matrices, and of rows and
   matrices in 8-bit integers.

   Common to them.  A token t chooses k of E experts; the (token, choice) pairs
   ordered by expert, then token, are the rows.  Element types are EMU_F32,
   EMU_BF16 (bfloat16) and EMU_F16 (binary16) of all matrices of a call;
   weights, their gradients and every sum are FP32, rounded once to the output's
   type.  FP32 products are those of emu_sgemm: three BF16 components of each
   operand, six component products, FP32 accumulation (so FP32 accuracy for
   2^-103 <= |a| < (2 - 2^-8) 2^127; a larger or non-finite entry makes its
   outputs NaN).  They raise no EMU_STATUS_* bits.
   Matrices are row-major with leading dimensions in elements, at any element's
   alignment; index arrays are int32.  Device pointers, ordered on the current
   stream, no host synchronisation (but where the workspace grows).  It is used by emu_moe_route
   (more than 64 tokens), emu_moe_balance (more than 256), emu_q4_gemm (a reduction that is
   split), the grouped products (16-bit operands that are copied to 16-byte alignment first,
   sums of few matrices in pieces) and emu_q8_gemm (operands that are copied, a reduction of one
   matrix that is split; at most 8 GiB); all but the first two do without it where it cannot
   grow (no memory beside what is held, EMU_WORKSPACE_LIMIT, a stream under capture).
   offsets: E + 1 entries, rows [offsets[e], offsets[e + 1]) belong to expert e
   (offsets[0] counts as 0); an expert may have none.  Rows from offsets[E] on
   belong to no expert: their outputs are zero and their inputs are not used.
   The values are read on the device and clamped to the rows that exist, so a
   router's result is passed on without the host's knowledge.
   rows: where given, row r of the product reads row rows[r] of X; an entry
   outside X (which may have no row at all) stands for a row of zeros.  Next to
   a W that is not finite, such a row of a product may be zeros or NaN.
   EMU_EINVAL (before any HIP call) for a bad type, negative sizes, a leading
   dimension below its row length, a NULL pointer to something that is not
   empty, or sizes beyond the limits given.  At most 2^24 - 1 tokens, 2^31 - 1
   rows and 2^30 - 1 columns; E at most 2^16; the leading dimensions of the
   grouped products at most 2^31 - 1. */
#define EMU_F32 0
#define EMU_BF16 1
#define EMU_F16 2

/* Router.  logits: T x E (ldl), 1 <= E <= 1024, 1 <= k <= min(E, 32).  ids
   (T x k): the experts with the k largest logits in descending order, the
   lowest index first among equal ones; -inf and NaN are never chosen, and -1
   fills up where fewer than k are left (weight 0, no row).  weights (T x k,
   FP32): exp(l - m) / S with m the token's largest logit and S the sum of the
   exponentials over the chosen experts (EMU_ROUTE_CHOSEN) or over all
   (EMU_ROUTE_ALL); experts at +inf share the weight.  offsets (E + 1); rows
   (T k): the token of each row, -1 from offsets[E] on; slots (T x k): the row
   of each choice, or -1.  The order is by expert, then token. */
#define EMU_ROUTE_CHOSEN 0
#define EMU_ROUTE_ALL 1
int emu_moe_route(int dtype, int64_t T, int E, int k, int scope, const void *logits, int64_t ldl,
                  int32_t *ids, float *weights, int32_t *offsets, int32_t *rows, int32_t *slots);
/* Gradient of the logits (T x E, ldd, fully written) from the gradient of the
   weights (T x k; the entries of ids = -1 are not used): w_j dw_j at the chosen
   experts, minus p_e sum_j w_j dw_j, p the softmax over the scope's set.
   logits are read in EMU_ROUTE_ALL only. */
int emu_moe_route_grad(int dtype, int64_t T, int E, int k, int scope, const void *logits, int64_t ldl,
                       const int32_t *ids, const float *weights, const float *dweights,
                       void *dlogits, int64_t ldd);

/* Y[t] = sum over j of weights[t, j] Z[slots[t, j]] (T x D, ldy); Z: R x D
   (ldz).  A slot outside Z adds nothing, whatever its weight.  weights NULL
   stands for ones (the gradient of reading token rows through `rows`).
   1 <= k <= 32. */
int emu_moe_combine(int dtype, int64_t T, int64_t D, int k, int64_t R, const void *Z, int64_t ldz,
                    const int32_t *slots, const float *weights, void *Y, int64_t ldy);
/* Its gradients: dZ[slots[t, j]] = weights[t, j] dY[t], zero for the rows with
   rows[r] < 0 (without tokens too); dweights[t, j] = <Z[slots[t, j]], dY[t]>, 0
   for a slot outside Z.
   slots and rows (R entries) as emu_moe_route gives them. */
int emu_moe_combine_grad(int dtype, int64_t T, int64_t D, int k, int64_t R, const void *dY,
                         int64_t lddy, const void *Z, int64_t ldz, const int32_t *slots,
                         const float *weights, const int32_t *rows, void *dZ, int64_t lddz,
                         float *dweights);

/* Y[r] = X[rows[r]] op(W[e(r)]) for the R rows of Y (R x N, ldy), op(W) K x N:
   W[e] starts at W + e stride and is K x N (ldw >= N) for transb 'N', N x K
   (ldw >= K) for 'T'.  X: XR x K (ldx); rows NULL stands for the row itself
   (XR >= R).  The gradient of the rows is the call with dY for X and the other
   transb. */
int emu_grouped_gemm(int dtype, char transb, int E, int64_t R, int64_t N, int64_t K, const void *X,
                     int64_t ldx, int64_t XR, const int32_t *rows, const void *W, int64_t ldw,
                     int64_t stride, const int32_t *offsets, void *Y, int64_t ldy);
/* Gradient of the matrices: dW[e] = sum over the rows r of e of X[rows[r]]^T
   dY[r], stored as W for the same transb (fully written; zeros for an expert
   without rows). */
int emu_grouped_wgrad(int dtype, char transb, int E, int64_t R, int64_t N, int64_t K, const void *X,
                      int64_t ldx, int64_t XR, const int32_t *rows, const void *dY, int64_t lddy,
                      const int32_t *offsets, void *dW, int64_t ldw, int64_t stride);

/* Matrices in 4 bits.  W is E x N x K, contiguous; byte j of a row of Q (K / 2
   bytes) holds entry 2 j in its low and 2 j + 1 in its high half, q in 0 .. 15.
   Each `group` (32, 64 or 128) entries along K share a scale s, and where mins
   is given an offset m, of the call's type (E x N x K / group):
   W = s (q - 8), or s q + m.  K is a multiple of the group.
   emu_q4_gemm: Y[r] = X[rows[r]] W[e(r)]^T for R rows ordered by expert as for
   emu_grouped_gemm (offsets NULL: E = 1, every row); made for few rows of each
   expert, where the bytes of Q bound it.  The products are formed with the exact
   integers 16 + q on matrix instructions and scaled per group in FP32; a sum that
   is not finite so (those integers leave FP32's range before W does, at entries of
   X above some 1e35) is formed again by the definition, in FP64.  So an infinite
   or NaN entry gives what the definition gives, for FP32 too. */
int emu_q4_gemm(int dtype, int E, int64_t R, int64_t N, int64_t K, int group, const void *X,
                int64_t ldx, int64_t XR, const int32_t *rows, const uint8_t *Q, const void *scales,
                const void *mins, const int32_t *offsets, void *Y, int64_t ldy);
/* Q and scales of `rows` rows of K entries (ldw): s = max |w| / 7 of the group,
   rounded to the call's type, q = 8 + the integer nearest w / s (ties to even)
   within -8 .. 7 (8 where s = 0; w must be finite). */
int emu_q4_pack(int dtype, int64_t rows, int64_t K, int group, const void *W, int64_t ldw, uint8_t *Q,
                void *scales);

/* The balance loss of a routing, for each of S sequences of tokens (1 <= S <= 65536).
   starts: S + 1 entries, sequence s has the tokens starts[s] to starts[s + 1] (starts[0]
   counts as 0; not descending, clamped to the T tokens that exist); the tokens from
   starts[S] on belong to none.  NULL: S = 1, every token.  logits and ids as
   emu_moe_route has them (entries of ids outside 0 .. E - 1 are not counted).  With p the
   softmax of a token's logits over all E experts (experts at +inf share it; -inf and NaN
   have none) and z the logarithm of its sum, n the tokens that have a logit above
   -inf, c_e the choices of expert e and C = sum c_e:
     loss[s] = E sum over e of (c_e / C) (1 / n) sum over tokens of p[t, e],
     zloss[s] = (1 / n) sum over tokens of z[t]^2,
     counts[s, e] = c_e,  tokens[s] = n
   (losses 0 where n or C is 0).  Workspace above 256 tokens. */
int emu_moe_balance(int dtype, int64_t T, int E, int k, int S, const void *logits, int64_t ldl,
                    const int32_t *ids, const int32_t *starts, float *loss, float *zloss,
                    int32_t *counts, int32_t *tokens);
/* Gradient of the logits (T x E, ldd, fully written; zeros for the tokens of no
   sequence) from the gradients of the losses (S entries; dzloss NULL: zeros), with the
   shares f_e = c_e / C taken as constant:
     p[t, e] (dloss E / n (f_e - sum over j of p[t, j] f_j) + dzloss 2 / n z[t]),
   0 where p is 0 or n is not positive.  counts (S x E) and tokens as emu_moe_balance
   gives them; where several processes share a batch, their sums. */
int emu_moe_balance_grad(int dtype, int64_t T, int E, int S, const void *logits, int64_t ldl,
                         const int32_t *counts, const int32_t *tokens, const int32_t *starts,
                         const float *dloss, const float *dzloss, void *dlogits, int64_t ldd);

/* Rows in 8-bit integers.  X: rows x K (ldx) of the call's type.  scales[r] =
   max |x| / 127 of the row, Q (rows x K, ldq) the integer nearest 127 x / max |x|, ties
   to even, -127 .. 127.  A row of zeros has scale 0; one with an infinity or a NaN
   has scale NaN and zeros.  emu_q8_unpack: X = scales[r] Q. */
int emu_q8_pack(int dtype, int64_t rows, int64_t K, const void *X, int64_t ldx, int8_t *Q, int64_t ldq,
                float *scales);
int emu_q8_unpack(int dtype, int64_t rows, int64_t K, const int8_t *Q, int64_t ldq, const float *scales,
                  void *X, int64_t ldx);
/* Products of rows in 8-bit integers with matrices in 8-bit integers: for R rows ordered
   by expert as for emu_grouped_gemm (offsets NULL: E = 1, every row)
     Y[r, n] = xscales[x] wscales[e, n] sum over k of X[x, k] W[e, n, k],
   e the row's expert and x its row of X, rows[r] (NULL: r itself).  dtype is Y's type.
   X: XR x K (ldx), xscales XR; W[e] starts at W + e stride and is N x K (ldw), wscales
   E x N.  Any integers, -128 too; the sums are exact (K <= 131071), each is rounded to
   FP32, multiplied there by wscales, then by xscales, and rounded to the type: the bits of
   a row of Y depend on its own operands alone, not on the other rows or the workspace.  A row
   of Y whose row of X does not exist is zeros.  Operands whose rows are not multiples of 16 bytes are
   copied to the workspace first where there are many rows; without workspace, and for
   few rows, they are read as they are.  A long reduction of one matrix (K from 1024 on) with
   few results is split over workgroups, whatever the alignment: the 32-bit sums, 2 to 16
   for a result, are in the workspace; without it the reduction is in one piece. */
int emu_q8_gemm(int dtype, int E, int64_t R, int64_t N, int64_t K, const int8_t *X, int64_t ldx,
                const float *xscales, int64_t XR, const int32_t *rows, const int8_t *W, int64_t ldw,
                int64_t stride, const float *wscales, const int32_t *offsets, void *Y, int64_t ldy);

/* Stream for subsequent calls (a hipStream_t); NULL selects the default
   stream.  Switching streams orders the new stream after the work already
   queued on the previous one (an event dependency, no host synchronisation),
   since every call uses the one workspace.  Streams under one capture are ordered
   in the same way, by an edge of its graph (of two captures at a time, the calls
   of each have to be on one stream).  A graph and what is outside of it are
   not: the caller orders the graph's launches, and calls outside follow the last
   ones outside.  A captured call must find the workspace grown already (by the
   same call before the capture; else EMU_ENOMEM, or it does without).  Its graph
   is good until emu_release_workspace: a workspace that captured calls use is kept
   until then when a larger one takes its place.  EMU_OK, or EMU_EHIP (the stream remains what it was) if
   a HIP call fails, or if the new stream is not under capture and would have to
   follow earlier work on one that now is. */
int emu_set_stream(void *hip_stream);

/* Projection constant of the FP64 split for subsequent emu_dgemm and
   emu_split_f64 calls: EMU_SPLIT_SYM (default) or EMU_SPLIT_LITERAL.
   EMU_EINVAL for any other value. */
int emu_set_split_mode(int mode);

/* Exponent scope of the FP64 split for subsequent emu_dgemm and emu_split_f64
   calls: EMU_SCOPE_OPERAND (default), EMU_SCOPE_ROWCOL or EMU_SCOPE_KBIN (see above).  In the
   ROWCOL scope the domain checks behind EMU_STATUS_RANGE apply to the scaled
   operands.  EMU_EINVAL for any other value. */
int emu_set_split_scope(int scope);

/* Synchronises the current stream, stores in *flags the EMU_STATUS_* bits
   accumulated by all calls since the previous emu_domain_status, and clears
   them.  EMU_EINVAL if flags is NULL. */
int emu_domain_status(unsigned *flags);

/* Message of the last failing call (empty string if none).  Owned by the
   library, valid until the next call. */
const char *emu_last_error(void);

/* Frees the workspace and those kept for graphs (synchronises the device
   first).  The next call allocates again. */
int emu_release_workspace(void);

/* Bytes currently held by the workspace (0 after emu_release_workspace), without
   those kept for graphs. */
int64_t emu_workspace_bytes(void);

/* Test hook: the FP32 split of Eq. (fp32split) as the GEMM consumes it.
   X is an R x Cc row-major FP32 device matrix (ldx).  as_b = 0 runs the
   A-operand pack (rows of X are GEMM rows), as_b = 1 the B-operand pack (X is
   K x N and is packed transposed).  comps (device, uint16 BF16 bit patterns)
   receives [3][R][Cc], plane-major, in X's own orientation, unpacked from the
   packed buffer.  Errors as above. */
int emu_split_f32(int64_t R, int64_t Cc, const float *X, int64_t ldx, int as_b, uint16_t *comps);

/* Test hook: the FP64 split of Eq. (fp64split) as the GEMM consumes it.
   X is R x Cc row-major FP64 (device, ldx); as_b as for emu_split_f32.
   slices (device) receives [6][R][Cc] BF16 bit patterns; v (device, int32[6])
   receives v^(r) = ceil(log2 max|X^(r)|) per level, INT32_MIN for a level
   whose residual is identically zero.  In the ROWCOL scope these are the
   slices and exponents of the scaled operand (rows of X scaled when as_b = 0,
   columns when as_b = 1). */
int emu_split_f64(int64_t R, int64_t Cc, const double *X, int64_t ldx, int as_b,
                  uint16_t *slices, int32_t *v);

/* Test hook: the weights of the ROWCOL scope.  X is R x Cc row-major FP64
   (device, ldx); s (device, int32) receives ceil(log2 max|x|) over each row
   (by_col = 0, R entries) or each column (by_col = 1, Cc entries), ignoring
   non-finite entries, 0 for a row or column without a nonzero finite entry.
   EMU_EINVAL for negative sizes, ldx < max(1, Cc), by_col not 0 or 1, or a
   NULL pointer with nonzero extent. */
int emu_scale_exponents(int64_t R, int64_t Cc, const double *X, int64_t ldx, int by_col,
                        int32_t *s);

/* Phase timing, the analog of the paper's runtime breakdown (Sec. 8.4):
   decomposition + packing versus the component-product GEMM with its
   reconstruction.  emu_profile_enable(1) creates a pool of HIP events for
   4096 calls (the only allocation, done here, outside any timed region); from
   then on every emu_sgemm / emu_dgemm records three events on its stream:
   before its split kernels, between them and its GEMM kernel, and after the
   GEMM kernel.  emu_profile_read synchronises the device, writes the split/pack
   and GEMM milliseconds of the profiled calls since the previous read, oldest
   first, into split_ms[i] and gemm_ms[i] for i < min(cap, *calls) (host arrays
   owned by the caller), stores the number of such calls in *calls and starts
   over.  Calls made while the pool is full are not profiled.
   emu_profile_enable(0) destroys the pool.  EMU_EINVAL if calls is NULL, or if
   cap > 0 and an array is NULL. */
int emu_profile_enable(int on);
int emu_profile_read(int64_t cap, double *split_ms, double *gemm_ms, int64_t *calls);

#ifdef __cplusplus
}
#endif

#endif /* EMU_H */
