"""The large forms of the grouped products: tiles of 256 x 256 and 128 x 128, one and
several to a workgroup, whole and partly filled, strided operands; operands on copies
without workspace; few rows in 16 bits 'T'.  Against 64 bits, summed on the GPU.
(test_kernel_choice asks which kernels these shapes launch.)"""
import pytest
import torch

import _moe as M
import _moe_shapes as S
from test_gpu_grouped import _case, _cuda

pytestmark = pytest.mark.gpu
HALVES = ["bf16", "f16"]


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


def _gathered(X, rows):
    if rows is None:
        return X.double()
    rows = rows.long()
    ok = (rows >= 0) & (rows < len(X))
    return X.double()[torch.where(ok, rows, 0)] * ok[:, None]


def _check_product(got, X, W, offsets, rows, K, dt):
    """One expert after the other: W (K x N) of each, `got` rows of none zero."""
    x, at = _gathered(X, rows), offsets.tolist()
    assert (got[at[-1]:] == 0).all()
    for e in range(len(W)):
        part = slice(at[e], at[e + 1])
        w = W[e].double()
        exact, size = x[part] @ w, x[part].abs() @ w.abs()
        off = (got[part].double() - exact).abs()
        assert torch.isfinite(got[part]).all() and (off <= M.product_bar(exact, size, K, dt)).all(), e


def _check_gradient(got, X, dY, offsets, rows, R, dt):
    """got: E x K x N."""
    x, at = _gathered(X, rows), offsets.tolist()
    for e in range(len(got)):
        part = slice(at[e], at[e + 1])
        x_e, y_e = x[part].T.contiguous(), dY[part].double()
        exact, size = x_e @ y_e, x_e.abs() @ y_e.abs()
        off = (got[e].double() - exact).abs()
        assert torch.isfinite(got[e]).all() and (off <= M.product_bar(exact, size, R, dt)).all(), e


def _wide(t, before, after, below=0):
    """t as a part of a larger tensor of NaN."""
    shape = (*t.shape[:-2], t.shape[-2] + below, t.shape[-1] + before + after)
    whole = torch.full(shape, float("nan"), dtype=t.dtype, device="cuda")
    part = whole[..., :t.shape[-2], before:before + t.shape[-1]]
    part.copy_(t)
    return part


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("R,E,N,K", S.TILES_256 + S.TILES_128)
def test_products(emu, kind, R, E, N, K, transb, gather):
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = (_cuda(t) for t in _case(R + N, R, E, N, K, dt, gather))
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    out = torch.full((R, N + 3), 9.0, dtype=dt, device="cuda")
    got = emu.grouped_gemm(X, w, offsets.int(), Y=out[:, 1:1 + N], transb=transb, rows=rows)
    _check_product(got, X, W, offsets, rows, K, dt)
    assert (out[:, 0] == 9).all() and (out[:, N + 1:] == 9).all()


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("R,E,N,K", [S.TILES_256[0], S.TILES_256[2], S.TILES_128[0]])
def test_strided_products(emu, kind, R, E, N, K, transb, gather):
    """Operands inside larger matrices of NaN, at 16 bytes."""
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = (_cuda(t) for t in _case(R + K, R, E, N, K, dt, gather))
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(_wide(X, 8, 16), _wide(w, 8, 8, 3), offsets.int(), transb=transb, rows=rows)
    _check_product(got, X, W, offsets, rows, K, dt)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("R,E,N,K", S.GRADIENTS_256 + S.GRADIENTS_128)
def test_gradients(emu, kind, R, E, N, K, transb, gather):
    dt = M.TYPES[kind]
    X, _, offsets, rows, dY = (_cuda(t) for t in _case(R + K, R, E, N, K, dt, gather))
    shape = (E, K + 1, N + 3) if transb == "N" else (E, N + 1, K + 3)
    dW = torch.full(shape, 9.0, dtype=dt, device="cuda")
    got = emu.grouped_wgrad(X, dY, offsets.int(), dW=dW[:, :-1, 1:-2], transb=transb, rows=rows)
    _check_gradient(got if transb == "N" else got.transpose(1, 2), X, dY, offsets, rows, R, dt)
    assert (dW[:, -1] == 9).all() and (dW[:, :, 0] == 9).all() and (dW[:, :, -2:] == 9).all()


@pytest.mark.parametrize("kind", HALVES)
def test_one_expert_has_every_row(emu, kind):
    """The runs of tiles that the XCDs get, where all but one expert are empty."""
    dt = M.TYPES[kind]
    for which in (0, 33, 63):
        R, E, N, K = S.GRADIENTS_256[0]
        X, _, _, _, dY = (_cuda(t) for t in _case(which, R, E, N, K, dt, False, 0.0))
        offsets = torch.zeros(E + 1, dtype=torch.int64)
        offsets[which + 1:] = R
        got = emu.grouped_wgrad(X, dY, offsets.int().cuda())
        _check_gradient(got, X, dY, offsets, None, R, dt)
        X, W, _, _, _ = (_cuda(t) for t in _case(which, 33000, E, 512, 128, dt, False, 0.0))
        offsets[which + 1:] = 33000
        _check_product(emu.grouped_gemm(X, W, offsets.int().cuda()), X, W, offsets, None, 128, dt)


@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("gather", [False, True])
def test_copies_and_without_workspace(emu, monkeypatch, kind, gather):
    """A product that is worth copies: on them, and where the workspace may not grow."""
    dt, (R, E, N, K) = M.TYPES[kind], S.COPIED
    X, W, offsets, rows, _ = (_cuda(t) for t in _case(R, R, E, N, K, dt, gather))
    _check_product(emu.grouped_gemm(X, W, offsets.int(), rows=rows), X, W, offsets, rows, K, dt)
    emu.release_workspace()
    monkeypatch.setenv("EMU_WORKSPACE_LIMIT", "4096")
    _check_product(emu.grouped_gemm(X, W, offsets.int(), rows=rows), X, W, offsets, rows, K, dt)
    assert emu.workspace_bytes() <= 4096


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("R,E,N,K", S.FEW_T)
def test_few_rows(emu, kind, R, E, N, K, gather):
    """Eight rows of an expert on average, unevenly: blocks of 1 to 16 rows, and many."""
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = (_cuda(t) for t in _case(R + N, R, E, N, K, dt, gather))
    w = W.transpose(1, 2).contiguous()
    _check_product(emu.grouped_gemm(X, w, offsets.int(), transb="T", rows=rows), X, W, offsets, rows, K, dt)
    offsets = torch.zeros(E + 1, dtype=torch.int64)
    offsets[E // 2 + 1:] = R                                # all at one expert
    X = X.nan_to_num()                                      # (the rows of no expert were NaN)
    got = emu.grouped_gemm(X, w, offsets.int().cuda(), transb="T", rows=rows)
    _check_product(got, X, W, offsets, rows, K, dt)
