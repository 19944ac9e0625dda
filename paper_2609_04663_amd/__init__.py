"""Python binding of libemu: FP32/FP64 GEMM emulated through BF16 component
products on AMD Instinct MI355X (gfx950), after arxiv 2609.04663.

Argument marshalling only: every step of the computation runs in the HIP
kernels of ``libemu.so`` (C ABI in ``include/emu.h``).  PyTorch supplies the
device memory and the stream; tensors must be CUDA (HIP) tensors, row-major
with unit stride in the last dimension.  There is no CPU fallback: if the
library is not built, importing the functions raises.

    sgemm(A, B, C=None)            -> C = A @ B, FP32, 3 components / 6 products
    dgemm(A, B, nprod, C=None)     -> C = A @ B, FP64, six slices / nprod products
    sgemm_ex / dgemm_ex(..., transa, transb, alpha, beta) -> BLAS form alpha op(A) op(B) + beta C
    split_f32(X, as_b=False)       -> int16 tensor [3, R, C] of BF16 bit patterns
    split_f64(X, as_b=False)       -> (int16 tensor [6, R, C], int32 tensor [6])
    set_split_scope(scope)         -> SCOPE_OPERAND (default) or SCOPE_ROWCOL weights
    scale_exponents(X, by_col)     -> int32 tensor of the ROWCOL weights
    domain_status()                -> EMU_STATUS_* bits accumulated since last call

Mixture-of-experts operators (float32, bfloat16 or float16; see emu.h):

    moe_route(logits, k, scope)    -> Routing(ids, weights, offsets, rows, slots)
    moe_route_grad(logits, ids, weights, dweights, scope) -> gradient of the logits
    moe_combine(Z, slots, weights) -> weighted sum of each token's rows of Z
    moe_combine_grad(dY, Z, slots, weights, rows) -> (dZ, dweights)
    grouped_gemm(X, W, offsets, transb, rows)    -> Y[r] = X[rows[r]] op(W[expert of r])
    grouped_wgrad(X, dY, offsets, transb, rows)  -> gradient of W
    q4_pack(W, group)              -> (Q, scales): W in 4 bits
    q4_gemm(X, Q, scales, mins, offsets, rows)   -> Y[r] = X[rows[r]] W[expert of r]^T
    moe_balance(logits, ids, starts) -> Balance(loss, zloss, counts, tokens) of each sequence
    moe_balance_grad(logits, counts, tokens, dloss, dzloss, starts) -> gradient of the logits
    q8_pack(X)                     -> (Q, scales): rows in 8-bit integers, a scale each
    q8_unpack(Q, scales, dtype)    -> what they stand for
    q8_gemm(X, xscales, W, wscales, offsets, rows, dtype) -> Y[r] = X[rows[r]] W[expert of r]^T
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libemu.so")

EMU_OK, EMU_EINVAL, EMU_EHIP, EMU_ENOMEM = 0, 1, 2, 3
STATUS_NAN, STATUS_RANGE, STATUS_SUBNORMAL, STATUS_OVERFLOW, STATUS_INEXACT = 1, 2, 4, 8, 16
STATUS_FALLBACK = 32
FALLBACK_NONE, FALLBACK_FP64 = 0, 1
SGEMM_SPLIT_PASS, SGEMM_SPLIT_STREAMED = 0, 1
SPLIT_SYM, SPLIT_LITERAL = 0, 1
SCOPE_OPERAND, SCOPE_ROWCOL, SCOPE_KBIN = 0, 1, 2
# the paper's product counts N_p(d), d = 3 .. 6 (Eq. fp64productcounts) ...
NPROD = (6, 10, 15, 21)
# ... and every depth d = 1 .. 11 of the selection S_d (Eq. product-selection)
NPROD_ALL = (1, 3, 6, 10, 15, 21, 26, 30, 33, 35, 36)

EXPORTS = ("emu_sgemm", "emu_dgemm", "emu_set_stream", "emu_set_split_mode",
           "emu_domain_status", "emu_last_error", "emu_release_workspace",
           "emu_workspace_bytes", "emu_split_f32", "emu_split_f64", "emu_profile_enable",
           "emu_profile_read", "emu_set_split_scope", "emu_scale_exponents", "emu_sgemm_ex",
           "emu_dgemm_ex", "emu_dgemm_noalloc", "emu_set_fallback", "emu_set_sgemm_split",
           "emu_moe_route", "emu_moe_route_grad", "emu_moe_combine", "emu_moe_combine_grad",
           "emu_grouped_gemm", "emu_grouped_wgrad", "emu_q4_gemm", "emu_q4_pack",
           "emu_moe_balance", "emu_moe_balance_grad", "emu_q8_pack", "emu_q8_unpack", "emu_q8_gemm")
ROUTE_SCOPES = {"chosen": 0, "all": 1}      # EMU_ROUTE_CHOSEN, EMU_ROUTE_ALL
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # EMU_F32, EMU_BF16, EMU_F16


class EmuError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libemu error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load libemu.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2609_04663_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        i64, p, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
        L.emu_sgemm.argtypes = [i64, i64, i64, p, i64, p, i64, p, i64]
        L.emu_dgemm.argtypes = [i64, i64, i64, p, i64, p, i64, p, i64, ci]
        L.emu_dgemm_noalloc.argtypes = [i64, i64, i64, p, i64, p, i64, p, i64, ci]
        L.emu_set_stream.argtypes = [p]
        L.emu_set_split_mode.argtypes = [ci]
        L.emu_set_split_scope.argtypes = [ci]
        L.emu_set_fallback.argtypes = [ci]
        L.emu_set_sgemm_split.argtypes = [ci]
        ch, f32, f64 = ctypes.c_char, ctypes.c_float, ctypes.c_double
        L.emu_sgemm_ex.argtypes = [ch, ch, i64, i64, i64, f32, p, i64, p, i64, f32, p, i64]
        L.emu_dgemm_ex.argtypes = [ch, ch, i64, i64, i64, f64, p, i64, p, i64, f64, p, i64, ci]
        L.emu_scale_exponents.argtypes = [i64, i64, p, i64, ci, p]
        L.emu_domain_status.argtypes = [ctypes.POINTER(ctypes.c_uint)]
        L.emu_last_error.restype = ctypes.c_char_p
        L.emu_workspace_bytes.restype = i64
        L.emu_split_f32.argtypes = [i64, i64, p, i64, ci, p]
        L.emu_split_f64.argtypes = [i64, i64, p, i64, ci, p, p]
        L.emu_profile_enable.argtypes = [ci]
        L.emu_profile_read.argtypes = [i64, p, p, ctypes.POINTER(ctypes.c_int64)]
        L.emu_moe_route.argtypes = [ci, i64, ci, ci, ci, p, i64, p, p, p, p, p]
        L.emu_moe_route_grad.argtypes = [ci, i64, ci, ci, ci, p, i64, p, p, p, p, i64]
        L.emu_moe_combine.argtypes = [ci, i64, i64, ci, i64, p, i64, p, p, p, i64]
        L.emu_moe_combine_grad.argtypes = [ci, i64, i64, ci, i64, p, i64, p, i64, p, p, p, p, i64, p]
        L.emu_grouped_gemm.argtypes = [ci, ch, ci, i64, i64, i64, p, i64, i64, p, p, i64, i64, p, p,
                                       i64]
        L.emu_grouped_wgrad.argtypes = [ci, ch, ci, i64, i64, i64, p, i64, i64, p, p, i64, p, p, i64,
                                        i64]
        L.emu_q4_gemm.argtypes = [ci, ci, i64, i64, i64, ci, p, i64, i64, p, p, p, p, p, p, i64]
        L.emu_q4_pack.argtypes = [ci, i64, i64, ci, p, i64, p, p]
        L.emu_moe_balance.argtypes = [ci, i64, ci, ci, ci, p, i64, p, p, p, p, p, p]
        L.emu_moe_balance_grad.argtypes = [ci, i64, ci, ci, p, i64, p, p, p, p, p, p, i64]
        L.emu_q8_pack.argtypes = [ci, i64, i64, p, i64, p, i64, p]
        L.emu_q8_unpack.argtypes = [ci, i64, i64, p, i64, p, p, i64]
        L.emu_q8_gemm.argtypes = [ci, ci, i64, i64, i64, p, i64, p, i64, p, p, i64, i64, p, p, p, i64]
        for name in ("emu_moe_route", "emu_moe_route_grad", "emu_moe_combine",
                     "emu_moe_combine_grad", "emu_grouped_gemm", "emu_grouped_wgrad",
                     "emu_q4_gemm", "emu_q4_pack", "emu_moe_balance", "emu_moe_balance_grad",
                     "emu_q8_pack", "emu_q8_unpack", "emu_q8_gemm"):
            getattr(L, name).restype = ci
        for name in ("emu_sgemm", "emu_dgemm", "emu_set_stream", "emu_set_split_mode",
                     "emu_domain_status", "emu_release_workspace", "emu_split_f32",
                     "emu_split_f64", "emu_profile_enable", "emu_profile_read",
                     "emu_set_split_scope", "emu_scale_exponents", "emu_sgemm_ex",
                     "emu_dgemm_ex", "emu_dgemm_noalloc", "emu_set_fallback",
                     "emu_set_sgemm_split"):
            getattr(L, name).restype = ci
        _lib = L
    return _lib


def _check(rc: int):
    if rc != EMU_OK:
        raise EmuError(rc, lib().emu_last_error().decode())


def _bind_stream(dev: torch.device):
    # the handle alone: a torch.cuda.Stream object costs 2 us to make
    _check(lib().emu_set_stream(torch._C._cuda_getCurrentRawStream(dev.index)))


def _layout(t: torch.Tensor, dtype, name: str):
    """dtype and row-major layout checks (metadata only, any device)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    # the stride of a dimension of extent 1 is never used (NumPy-made tensors
    # of shape (1, n) can carry a row stride of 1)
    shape, stride = t.shape, t.stride()
    if (len(shape) != 2 or (shape[1] > 1 and stride[1] != 1)
            or (shape[0] > 1 and stride[0] < max(1, shape[1]))):
        raise ValueError(f"{name} must be a row-major 2-D tensor with unit column stride")
    return t


def _on_gpu(*named):
    for name, t in named:
        if not t.is_cuda:
            raise TypeError(f"{name} must be a GPU tensor")


def _mat(t: torch.Tensor, dtype, name: str):
    _layout(t, dtype, name)
    _on_gpu((name, t))
    return t


def _out(C, M: int, N: int, dtype, device):
    """The output C: allocated when None, else checked to be M x N (the
    library writes M rows of ldc elements: a smaller C would be overrun)."""
    if C is None:
        return torch.empty((M, N), dtype=dtype, device=device)
    _layout(C, dtype, "C")
    if tuple(C.shape) != (M, N):
        raise ValueError(f"C must be {M} x {N}, got {tuple(C.shape)}")
    return C


def _ld(t: torch.Tensor) -> int:
    rows, cols = t.shape
    if rows <= 1:
        return max(1, cols)
    return max(1, t.stride(0), cols)


def sgemm(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor | None = None) -> torch.Tensor:
    _layout(A, torch.float32, "A")
    _layout(B, torch.float32, "B")
    M, K = A.shape
    K2, N = B.shape
    if K != K2:
        raise ValueError("inner dimensions differ")
    C = _out(C, M, N, torch.float32, A.device)
    _on_gpu(("A", A), ("B", B), ("C", C))
    _bind_stream(A.device)
    _check(lib().emu_sgemm(M, N, K, A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), C.data_ptr(),
                           _ld(C)))
    return C


def dgemm(A: torch.Tensor, B: torch.Tensor, nprod: int,
          C: torch.Tensor | None = None) -> torch.Tensor:
    _layout(A, torch.float64, "A")
    _layout(B, torch.float64, "B")
    M, K = A.shape
    K2, N = B.shape
    if K != K2:
        raise ValueError("inner dimensions differ")
    C = _out(C, M, N, torch.float64, A.device)
    _on_gpu(("A", A), ("B", B), ("C", C))
    _bind_stream(A.device)
    _check(lib().emu_dgemm(M, N, K, A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), C.data_ptr(),
                           _ld(C), int(nprod)))
    return C


def dgemm_noalloc(A: torch.Tensor, B: torch.Tensor, nprod: int, C: torch.Tensor) -> torch.Tensor:
    """dgemm into a caller-supplied C without any device allocation by the
    library (its fixed scratch; see emu_dgemm_noalloc in emu.h)."""
    _layout(A, torch.float64, "A")
    _layout(B, torch.float64, "B")
    M, K = A.shape
    K2, N = B.shape
    if K != K2:
        raise ValueError("inner dimensions differ")
    if C is None:
        raise ValueError("dgemm_noalloc needs C")
    C = _out(C, M, N, torch.float64, A.device)
    _on_gpu(("A", A), ("B", B), ("C", C))
    _bind_stream(A.device)
    _check(lib().emu_dgemm_noalloc(M, N, K, A.data_ptr(), _ld(A), B.data_ptr(), _ld(B),
                                   C.data_ptr(), _ld(C), int(nprod)))
    return C


def _op_shape(X: torch.Tensor, trans: str):
    if trans not in ("N", "T"):
        raise ValueError("trans must be 'N' or 'T'")
    return (X.shape[1], X.shape[0]) if trans == "T" else tuple(X.shape)


def _gemm_ex(fn, dtype, A, B, C, transa, transb, alpha, beta, extra=()):
    _layout(A, dtype, "A")
    _layout(B, dtype, "B")
    M, K = _op_shape(A, transa)
    K2, N = _op_shape(B, transb)
    if K != K2:
        raise ValueError("inner dimensions differ")
    if C is None and beta != 0:
        raise ValueError("beta != 0 needs C")
    C = _out(C, M, N, dtype, A.device)
    _on_gpu(("A", A), ("B", B), ("C", C))
    _bind_stream(A.device)
    _check(fn(transa.encode(), transb.encode(), M, N, K, alpha, A.data_ptr(), _ld(A),
              B.data_ptr(), _ld(B), beta, C.data_ptr(), _ld(C), *extra))
    return C


def sgemm_ex(A, B, C=None, transa="N", transb="N", alpha=1.0, beta=0.0):
    """C = alpha op(A) op(B) + beta C in FP32 (A, B as stored; see emu.h)."""
    return _gemm_ex(lib().emu_sgemm_ex, torch.float32, A, B, C, transa, transb, float(alpha),
                    float(beta))


def dgemm_ex(A, B, nprod, C=None, transa="N", transb="N", alpha=1.0, beta=0.0):
    """C = alpha op(A) op(B) + beta C in FP64 with nprod retained products."""
    return _gemm_ex(lib().emu_dgemm_ex, torch.float64, A, B, C, transa, transb, float(alpha),
                    float(beta), (int(nprod),))


# ---------------------------------------------------------------------------
# Mixture-of-experts operators.

class Routing(NamedTuple):
    """moe_route's result: T tokens, k choices, E experts (see emu_moe_route)."""
    ids: torch.Tensor        # T x k, the experts in descending order, -1 for none
    weights: torch.Tensor    # T x k, float32
    offsets: torch.Tensor    # E + 1, first row of each expert
    rows: torch.Tensor       # T k, the token of each row, -1 past the last
    slots: torch.Tensor      # T x k, the row of each choice, -1 for none


def _float_mat(t, name: str, like=None) -> int:
    """The element code of a row-major matrix of a supported type."""
    if type(t) is torch.Tensor and t.dim() == 2 and t.is_contiguous():      # the cheaper look
        code = _DTYPES.get(t.dtype)
        if code is not None and (like is None or t.dtype is like.dtype):
            return code
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    _layout(t, t.dtype if like is None else like.dtype, name)
    return code


def _packed(t, name: str, dtype, shape):
    """A contiguous tensor of this type and shape (a tuple)."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {' x '.join(map(str, shape))}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _experts(t, name: str, dtype):
    """E, rows, columns, leading dimension and stride of E row-major matrices."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must be a 3-D tensor")
    E, a, b = t.shape
    ld = t.stride(1) if a > 1 else b
    if (b > 1 and t.stride(2) != 1) or ld < b or (E > 1 and t.stride(0) < 0):
        raise ValueError(f"{name} must hold row-major matrices with unit column stride")
    return E, a, b, max(1, ld), t.stride(0) if E > 1 else 0


def _ptr(t):
    return None if t is None else t.data_ptr()


def _launch(fn, device, *args):
    """One call on the current stream of the operands' device."""
    at = device.index
    if at == torch._C._cuda_getDevice():
        rc = lib().emu_set_stream(torch._C._cuda_getCurrentRawStream(at))
        if rc == EMU_OK:
            rc = fn(*args)
    else:
        with torch.cuda.device(device):
            _bind_stream(device)
            rc = fn(*args)
    if rc != EMU_OK:
        _check(rc)


def _same_gpu(*named):
    """Every tensor that is given is on the first one's GPU."""
    first, lead = named[0]
    at = lead.get_device()                      # (device objects cost more to compare)
    for _, t in named:
        if t is not None and t.get_device() != at:
            break
    else:
        if at >= 0:
            return
    device = lead.device
    for name, t in named:
        if t is None:
            continue
        if not t.is_cuda:
            raise TypeError(f"{name} must be a GPU tensor")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, {first} on {device}")


def _scope(scope: str) -> int:
    if scope not in ROUTE_SCOPES:
        raise ValueError("scope must be 'chosen' or 'all'")
    return ROUTE_SCOPES[scope]


def moe_route(logits: torch.Tensor, k: int, scope: str = "chosen") -> Routing:
    """The k experts of each token, their softmax weights over the chosen
    experts or over all, and the rows' order by expert (see emu_moe_route)."""
    code, how = _float_mat(logits, "logits"), _scope(scope)
    T, E = logits.shape
    _same_gpu(("logits", logits))
    dev = logits.device
    # tensors of their own: a caller may keep one, or change one in place while autograd
    # holds another (as parts of one allocation 1 us less)
    ids = logits.new_empty((T, k), dtype=torch.int32)
    slots, weights = torch.empty_like(ids), torch.empty_like(ids, dtype=torch.float32)
    rows, offsets = ids.new_empty(T * k), ids.new_empty(E + 1)
    _launch(lib().emu_moe_route, dev, code, T, E, k, how, logits.data_ptr(), _ld(logits),
            ids.data_ptr(), weights.data_ptr(), offsets.data_ptr(), rows.data_ptr(),
            slots.data_ptr())
    return Routing(ids, weights, offsets, rows, slots)


def moe_route_grad(logits, ids, weights, dweights, scope: str = "chosen") -> torch.Tensor:
    """Gradient of the logits from the gradient of moe_route's weights."""
    code, how = _float_mat(logits, "logits"), _scope(scope)
    T, E = logits.shape
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be a T x k tensor")
    k = ids.shape[1]
    _packed(ids, "ids", torch.int32, (T, k))
    _packed(weights, "weights", torch.float32, (T, k))
    _packed(dweights, "dweights", torch.float32, (T, k))
    _same_gpu(("logits", logits), ("ids", ids), ("weights", weights), ("dweights", dweights))
    out = logits.new_empty((T, E))
    _launch(lib().emu_moe_route_grad, logits.device, code, T, E, k, how, logits.data_ptr(),
            _ld(logits), ids.data_ptr(), weights.data_ptr(), dweights.data_ptr(), out.data_ptr(), E)
    return out


def _slots(slots, weights):
    if not isinstance(slots, torch.Tensor) or slots.dim() != 2:
        raise ValueError("slots must be a T x k tensor")
    T, k = slots.shape
    _packed(slots, "slots", torch.int32, (T, k))
    if weights is not None:
        _packed(weights, "weights", torch.float32, (T, k))
    return T, k


def moe_combine(Z, slots, weights=None, Y=None) -> torch.Tensor:
    """Y[t] = sum over j of weights[t, j] Z[slots[t, j]] (weights None: ones)."""
    code = _float_mat(Z, "Z")
    T, k = _slots(slots, weights)
    R, D = Z.shape
    Y = _rows_out(Y, T, D, Z, "Y")
    _same_gpu(("Z", Z), ("slots", slots), ("weights", weights), ("Y", Y))
    _launch(lib().emu_moe_combine, Z.device, code, T, D, k, R, Z.data_ptr(), _ld(Z),
            slots.data_ptr(), _ptr(weights), Y.data_ptr(), _ld(Y))
    return Y


def moe_combine_grad(dY, Z, slots, weights, rows):
    """(dZ, dweights): the gradients of moe_combine; rows as moe_route gives them."""
    code = _float_mat(Z, "Z")
    _float_mat(dY, "dY", Z)
    if weights is None:
        raise TypeError("weights must be a torch.Tensor")
    T, k = _slots(slots, weights)
    R, D = Z.shape
    if tuple(dY.shape) != (T, D):
        raise ValueError(f"dY must be {T} x {D}, got {tuple(dY.shape)}")
    _packed(rows, "rows", torch.int32, (R,))
    _same_gpu(("Z", Z), ("dY", dY), ("slots", slots), ("weights", weights), ("rows", rows))
    dZ, dw = Z.new_empty((R, D)), torch.empty_like(weights)
    _launch(lib().emu_moe_combine_grad, Z.device, code, T, D, k, R, dY.data_ptr(), _ld(dY),
            Z.data_ptr(), _ld(Z), slots.data_ptr(), weights.data_ptr(), rows.data_ptr(),
            dZ.data_ptr(), max(1, D), dw.data_ptr())
    return dZ, dw


def _rows_out(Y, R: int, N: int, like, name: str):
    """An output of R rows: allocated when None, else checked to be R x N."""
    if Y is None:
        return like.new_empty((R, N))
    _float_mat(Y, name, like)
    if tuple(Y.shape) != (R, N):
        raise ValueError(f"{name} must be {R} x {N}, got {tuple(Y.shape)}")
    return Y


def _grouping(X, offsets, rows, E: int, R=None) -> int:
    """The number of rows of a grouped product, its index arrays checked."""
    if offsets is not None:
        _packed(offsets, "offsets", torch.int32, (E + 1,))
    if rows is not None:
        if not isinstance(rows, torch.Tensor) or rows.dim() != 1:
            raise ValueError("rows must be a 1-D tensor")
        _packed(rows, "rows", torch.int32, rows.shape)
    n = X.shape[0] if rows is None else rows.shape[0]
    if R is not None and n != R:
        raise ValueError(f"{n} rows of X for {R} rows of the product")
    return n


def _transb(transb: str) -> bool:
    if transb not in ("N", "T"):
        raise ValueError("transb must be 'N' or 'T'")
    return transb == "T"


def grouped_gemm(X, W, offsets, Y=None, transb: str = "N", rows=None) -> torch.Tensor:
    """Y[r] = X[r] op(W[e(r)]), or X[rows[r]]; rows ordered by expert, expert e
    has the rows offsets[e] to offsets[e + 1].  W: E x K x N ("N") or E x N x K
    ("T")."""
    code, tb = _float_mat(X, "X"), _transb(transb)
    E, a, b, ldw, stride = _experts(W, "W", X.dtype)
    N, K = (a, b) if tb else (b, a)
    if X.shape[1] != K:
        raise ValueError("inner dimensions differ")
    if offsets is None:
        raise TypeError("offsets must be a torch.Tensor")
    R = _grouping(X, offsets, rows, E)
    Y = _rows_out(Y, R, N, X, "Y")
    _same_gpu(("X", X), ("W", W), ("offsets", offsets), ("rows", rows), ("Y", Y))
    _launch(lib().emu_grouped_gemm, X.device, code, transb.encode(), E, R, N, K, X.data_ptr(),
            _ld(X), X.shape[0], _ptr(rows), W.data_ptr(), ldw, stride, offsets.data_ptr(),
            Y.data_ptr(), _ld(Y))
    return Y


def grouped_wgrad(X, dY, offsets, dW=None, transb: str = "N", rows=None) -> torch.Tensor:
    """dW[e] = sum over the rows r of expert e of X[r]^T dY[r] (X[rows[r]] with
    rows), E x K x N for "N", its transpose E x N x K for "T"."""
    code, tb = _float_mat(X, "X"), _transb(transb)
    _float_mat(dY, "dY", X)
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("offsets must be a 1-D tensor of E + 1 entries")
    E = offsets.shape[0] - 1
    R, N, K = dY.shape[0], dY.shape[1], X.shape[1]
    _grouping(X, offsets, rows, E, R)
    shape = (E, N, K) if tb else (E, K, N)
    if dW is None:
        dW = X.new_empty(shape)
    elif tuple(dW.shape) != shape:
        raise ValueError(f"dW must be {' x '.join(map(str, shape))}, got {tuple(dW.shape)}")
    _, _, _, ldw, stride = _experts(dW, "dW", X.dtype)
    _same_gpu(("X", X), ("dY", dY), ("offsets", offsets), ("rows", rows), ("dW", dW))
    _launch(lib().emu_grouped_wgrad, X.device, code, transb.encode(), E, R, N, K, X.data_ptr(),
            _ld(X), X.shape[0], _ptr(rows), dY.data_ptr(), _ld(dY), offsets.data_ptr(),
            dW.data_ptr(), ldw, stride)
    return dW


def q4_pack(W: torch.Tensor, group: int = 64):
    """(Q, scales) of E x N x K (or N x K) matrices: 4-bit entries, two to a byte
    along K, and a scale for each group (see emu_q4_pack)."""
    if not isinstance(W, torch.Tensor) or W.dim() not in (2, 3):
        raise ValueError("W must be a 2-D or 3-D tensor")
    lead, K = W.shape[:-1], W.shape[-1]
    flat = W.reshape(lead.numel(), K)
    code = _float_mat(flat, "W")
    if group not in (32, 64, 128) or K % group:
        raise ValueError("group must be 32, 64 or 128 and divide K")
    _same_gpu(("W", W))
    Q = torch.empty((*lead, K // 2), dtype=torch.uint8, device=W.device)
    scales = torch.empty((*lead, K // group), dtype=W.dtype, device=W.device)
    _launch(lib().emu_q4_pack, W.device, code, flat.shape[0], K, group, flat.data_ptr(), _ld(flat),
            Q.data_ptr(), scales.data_ptr())
    return Q, scales


def q4_gemm(X, Q, scales, mins=None, offsets=None, rows=None, Y=None) -> torch.Tensor:
    """Y[r] = X[r] W[e(r)]^T (X[rows[r]] with rows), W in 4 bits as q4_pack gives
    it, with mins as W = scales q + mins.  Q: E x N x K/2; without offsets one
    matrix (E = 1, or Q N x K/2) serves every row."""
    code = _float_mat(X, "X")
    if not isinstance(Q, torch.Tensor) or Q.dim() not in (2, 3):
        raise ValueError("Q must be a 2-D or 3-D tensor")
    E, N, half = (1, *Q.shape) if Q.dim() == 2 else Q.shape
    K = X.shape[1]
    if 2 * half != K:
        raise ValueError("inner dimensions differ")
    if offsets is None and E != 1:
        raise ValueError("more than one matrix needs offsets")
    _packed(Q, "Q", torch.uint8, Q.shape)
    groups = scales.shape[-1] if isinstance(scales, torch.Tensor) and scales.dim() > 0 else 0
    group = K // groups if groups else 0
    if K and (group not in (32, 64, 128) or group * groups != K):
        raise ValueError("scales must have K / 32, K / 64 or K / 128 columns")
    _packed(scales, "scales", X.dtype, (*Q.shape[:-1], groups))
    if mins is not None:
        _packed(mins, "mins", X.dtype, scales.shape)
    R = _grouping(X, offsets, rows, E)
    Y = _rows_out(Y, R, N, X, "Y")
    _same_gpu(("X", X), ("Q", Q), ("scales", scales), ("mins", mins), ("offsets", offsets),
              ("rows", rows), ("Y", Y))
    _launch(lib().emu_q4_gemm, X.device, code, E, R, N, K, group or 32, X.data_ptr(), _ld(X),
            X.shape[0], _ptr(rows), Q.data_ptr(), scales.data_ptr(), _ptr(mins), _ptr(offsets),
            Y.data_ptr(), _ld(Y))
    return Y


class Balance(NamedTuple):
    """moe_balance's result for S sequences and E experts (see emu_moe_balance)."""
    loss: torch.Tensor       # S, float32: E sum_e f_e P_e
    zloss: torch.Tensor      # S, float32: the mean squared log of the softmax's sum
    counts: torch.Tensor     # S x E, int32, the choices of each expert
    tokens: torch.Tensor     # S, int32, the tokens with a logit above -inf


def _sequences(starts) -> int:
    """The number of sequences of the starts (None: one, all tokens)."""
    if starts is None:
        return 1
    if not isinstance(starts, torch.Tensor) or starts.dim() != 1 or starts.shape[0] < 2:
        raise ValueError("starts must be a 1-D tensor of S + 1 entries")
    _packed(starts, "starts", torch.int32, starts.shape)
    return starts.shape[0] - 1


def moe_balance(logits, ids, starts=None) -> Balance:
    """The balance loss, the squared log of the softmax's sum and the experts' counts of
    a routing; of each sequence, whose tokens are starts[s] to starts[s + 1]."""
    code, S = _float_mat(logits, "logits"), _sequences(starts)
    T, E = logits.shape
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be a T x k tensor")
    k = ids.shape[1]
    _packed(ids, "ids", torch.int32, (T, k))
    _same_gpu(("logits", logits), ("ids", ids), ("starts", starts))
    loss = logits.new_empty(S, dtype=torch.float32)
    zloss, tokens, counts = torch.empty_like(loss), ids.new_empty(S), ids.new_empty((S, E))
    _launch(lib().emu_moe_balance, logits.device, code, T, E, k, S, logits.data_ptr(), _ld(logits),
            ids.data_ptr(), _ptr(starts), loss.data_ptr(), zloss.data_ptr(), counts.data_ptr(),
            tokens.data_ptr())
    return Balance(loss, zloss, counts, tokens)


def moe_balance_grad(logits, counts, tokens, dloss, dzloss=None, starts=None) -> torch.Tensor:
    """Gradient of the logits from the gradients of moe_balance's losses (dzloss
    None: zeros); counts and tokens as moe_balance gives them, or sums of several."""
    code, S = _float_mat(logits, "logits"), _sequences(starts)
    T, E = logits.shape
    _packed(counts, "counts", torch.int32, (S, E))
    _packed(tokens, "tokens", torch.int32, (S,))
    _packed(dloss, "dloss", torch.float32, (S,))
    if dzloss is not None:
        _packed(dzloss, "dzloss", torch.float32, (S,))
    _same_gpu(("logits", logits), ("counts", counts), ("tokens", tokens), ("dloss", dloss),
              ("dzloss", dzloss), ("starts", starts))
    out = logits.new_empty((T, E))
    _launch(lib().emu_moe_balance_grad, logits.device, code, T, E, S, logits.data_ptr(), _ld(logits),
            counts.data_ptr(), tokens.data_ptr(), _ptr(starts), dloss.data_ptr(), _ptr(dzloss),
            out.data_ptr(), E)
    return out


def _int8_mat(t, name: str):
    if type(t) is torch.Tensor and t.dtype is torch.int8 and t.dim() == 2 and t.is_contiguous():
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    return _layout(t, torch.int8, name)


def _shaped(t, dtype):
    """A contiguous tensor of t's shape (empty_like is the cheapest)."""
    return torch.empty_like(t, dtype=dtype) if t.is_contiguous() else t.new_empty(t.shape, dtype=dtype)


def _code_of(dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    return code


def q8_pack(X: torch.Tensor):
    """(Q, scales) of the rows of X (two or more dimensions): 8-bit integers of X's
    shape and a float32 scale for each row (see emu_q8_pack)."""
    if not isinstance(X, torch.Tensor) or X.dim() < 2:
        raise ValueError("X must be a tensor of two or more dimensions")
    lead, K = X.shape[:-1], X.shape[-1]
    flat = X if X.dim() == 2 else X.reshape(lead.numel(), K)
    code = _float_mat(flat, "X")
    _same_gpu(("X", X))
    Q, scales = _shaped(X, torch.int8), X.new_empty(lead, dtype=torch.float32)
    _launch(lib().emu_q8_pack, X.device, code, flat.shape[0], K, flat.data_ptr(), _ld(flat), Q.data_ptr(),
            max(1, K), scales.data_ptr())
    return Q, scales


def q8_unpack(Q, scales, dtype=torch.bfloat16) -> torch.Tensor:
    """What q8_pack's integers stand for, scales Q, in this type."""
    code = _code_of(dtype)
    if not isinstance(Q, torch.Tensor) or Q.dim() < 2:
        raise ValueError("Q must be a tensor of two or more dimensions")
    lead, K = Q.shape[:-1], Q.shape[-1]
    flat = Q if Q.dim() == 2 else Q.reshape(lead.numel(), K)
    _int8_mat(flat, "Q")
    _packed(scales, "scales", torch.float32, lead)
    _same_gpu(("Q", Q), ("scales", scales))
    X = _shaped(Q, dtype)
    _launch(lib().emu_q8_unpack, Q.device, code, flat.shape[0], K, flat.data_ptr(), _ld(flat),
            scales.data_ptr(), X.data_ptr(), max(1, K))
    return X


def q8_gemm(X, xscales, W, wscales, offsets=None, rows=None, dtype=torch.bfloat16, Y=None) -> torch.Tensor:
    """Y[r] = X[r] W[e(r)]^T (X[rows[r]] with rows), X and W in 8 bits as q8_pack
    gives them, Y in `dtype` (with Y given: its own).  W: E x N x K; without
    offsets one matrix (E = 1, or W N x K) serves every row."""
    _int8_mat(X, "X")
    if not isinstance(W, torch.Tensor) or W.dim() not in (2, 3):
        raise ValueError("W must be a 2-D or 3-D tensor")
    if W.dtype is torch.int8 and W.is_contiguous():
        E, N, K = (1, *W.shape) if W.dim() == 2 else W.shape
        ldw, stride = max(1, K), N * K
    else:
        E, N, K, ldw, stride = _experts(W if W.dim() == 3 else W[None], "W", torch.int8)
    if X.shape[1] != K:
        raise ValueError("inner dimensions differ")
    if offsets is None and E != 1:
        raise ValueError("more than one matrix needs offsets")
    _packed(xscales, "xscales", torch.float32, (X.shape[0],))
    _packed(wscales, "wscales", torch.float32, W.shape[:-1])
    R = _grouping(X, offsets, rows, E)
    if Y is None:
        code = _code_of(dtype)
        Y = X.new_empty((R, N), dtype=dtype)
    else:
        code = _float_mat(Y, "Y")
        if tuple(Y.shape) != (R, N):
            raise ValueError(f"Y must be {R} x {N}, got {tuple(Y.shape)}")
    _same_gpu(("X", X), ("xscales", xscales), ("W", W), ("wscales", wscales), ("offsets", offsets),
              ("rows", rows), ("Y", Y))
    _launch(lib().emu_q8_gemm, X.device, code, E, R, N, K, X.data_ptr(), _ld(X), xscales.data_ptr(),
            X.shape[0], _ptr(rows), W.data_ptr(), ldw, stride, wscales.data_ptr(), _ptr(offsets),
            Y.data_ptr(), _ld(Y))
    return Y


def split_f32(X: torch.Tensor, as_b: bool = False) -> torch.Tensor:
    _mat(X, torch.float32, "X")
    R, Cc = X.shape
    out = torch.empty((3, R, Cc), dtype=torch.int16, device=X.device)
    _bind_stream(X.device)
    _check(lib().emu_split_f32(R, Cc, X.data_ptr(), _ld(X), int(as_b), out.data_ptr()))
    return out


def split_f64(X: torch.Tensor, as_b: bool = False):
    _mat(X, torch.float64, "X")
    R, Cc = X.shape
    out = torch.empty((6, R, Cc), dtype=torch.int16, device=X.device)
    v = torch.empty(6, dtype=torch.int32, device=X.device)
    _bind_stream(X.device)
    _check(lib().emu_split_f64(R, Cc, X.data_ptr(), _ld(X), int(as_b), out.data_ptr(),
                               v.data_ptr()))
    return out, v


def set_split_mode(mode: int):
    _check(lib().emu_set_split_mode(int(mode)))


def set_sgemm_split(mode: int):
    """SGEMM_SPLIT_PASS (split kernel, then the product kernel) or
    SGEMM_SPLIT_STREAMED (the product kernel splits its own k-blocks)."""
    _check(lib().emu_set_sgemm_split(int(mode)))


def set_fallback(mode: int):
    """FALLBACK_NONE (the paper's behaviour) or FALLBACK_FP64 (see emu.h)."""
    _check(lib().emu_set_fallback(int(mode)))


def set_split_scope(scope: int):
    """SCOPE_OPERAND (the paper's split) or SCOPE_ROWCOL (row/column weights)."""
    _check(lib().emu_set_split_scope(int(scope)))


def scale_exponents(X: torch.Tensor, by_col: bool = False) -> torch.Tensor:
    _mat(X, torch.float64, "X")
    R, Cc = X.shape
    out = torch.empty(Cc if by_col else R, dtype=torch.int32, device=X.device)
    _bind_stream(X.device)
    _check(lib().emu_scale_exponents(R, Cc, X.data_ptr(), _ld(X), int(by_col), out.data_ptr()))
    return out


def domain_status() -> int:
    f = ctypes.c_uint(0)
    _check(lib().emu_domain_status(ctypes.byref(f)))
    return int(f.value)


def profile_enable(on: bool = True):
    """Record split/pack and GEMM phase times of every call (see emu.h)."""
    _check(lib().emu_profile_enable(int(on)))


def profile_read(cap: int = 4096):
    """Per-call (split_ms, gemm_ms) lists of the profiled calls since the last
    read, oldest first; synchronises."""
    s = (ctypes.c_double * cap)()
    g = (ctypes.c_double * cap)()
    n = ctypes.c_int64()
    _check(lib().emu_profile_read(cap, s, g, ctypes.byref(n)))
    k = min(cap, int(n.value))
    return list(s[:k]), list(g[:k])


def release_workspace():
    _check(lib().emu_release_workspace())


def workspace_bytes() -> int:
    return int(lib().emu_workspace_bytes())
