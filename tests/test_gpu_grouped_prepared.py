"""Grouped products whose operands are prepared first: 16-bit matrices at odd
elements or of odd extents that are worth a copy, and gradients of few tiles whose
experts' rows are summed in pieces; against 64 bits."""
import math

import pytest
import torch

import _moe as M
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


def _inside(t, before, after):
    """t as a part of a wider tensor of NaN, `before` elements from its rows' starts."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + before + after), math.nan, dtype=t.dtype)
    wide[..., before:before + t.shape[-1]] = t
    return wide.cuda()[..., before:before + t.shape[-1]]


@pytest.mark.parametrize("gather", ["no", "few", "many"])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("R,E,N,K,x,w", [
    (4000, 2, 1000, 2001, 0, 0), (6100, 5, 1031, 1024, 0, 0), (5000, 1, 1024, 2048, 3, 0),
    (5000, 3, 1024, 2048, 0, 5), (9000, 4, 2050, 70, 1, 2), (5000, 2, 2001, 1500, 4, 8)])
def test_product(emu, kind, R, E, N, K, x, w, transb, gather):
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = _case(R + N, R, E, N, K, dt, gather != "no")
    if gather == "many":                                # more rows of X than are read
        X = torch.cat((X, torch.full((R + 100 - len(X), K), math.nan, dtype=dt)))
        rows[1] = len(X) + 5
    Y, S = M.grouped(X, W, offsets, rows)
    wt = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(_inside(X, x, 1) if x else X.cuda(), _inside(wt, w, 3) if w else wt.cuda(),
                           offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got, Y, M.product_bar(Y, S, K, dt))


@pytest.mark.parametrize("gather", ["no", "few", "many"])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("R,E,N,K,x,y", [
    (3000, 2, 700, 1001, 0, 0), (6100, 5, 1031, 512, 0, 0), (5000, 1, 600, 520, 3, 0), (4500, 3, 512, 800, 0, 5)])
def test_gradient_of_the_matrices(emu, kind, R, E, N, K, x, y, transb, gather):
    dt = M.TYPES[kind]
    X, _, offsets, rows, dY = _case(R + K, R, E, N, K, dt, gather != "no")
    if gather == "many":
        X = torch.cat((X, torch.full((R + 100 - len(X), K), math.nan, dtype=dt)))
        rows[1] = len(X) + 5
    ref, S = M.wgrad(X, dY, offsets, rows)
    got = emu.grouped_wgrad(_inside(X, x, 2) if x else X.cuda(), _inside(dY, y, 1) if y else dY.cuda(),
                            offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got if transb == "N" else got.transpose(1, 2), ref, M.product_bar(ref, S, R, dt))


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K", [
    (600, 1, 64, 64), (5000, 4, 86, 338), (3000, 2, 256, 128), (20000, 1, 130, 131), (9000, 13, 40, 200),
    (4100, 1, 1, 1), (40000, 8, 160, 96), (6000, 3, 512, 512)])
def test_gradient_in_pieces(emu, kind, R, E, N, K, gather):
    """A few more roundings: the pieces' sums are added one after the other."""
    dt = M.TYPES[kind]
    X, _, offsets, rows, dY = _case(R + K, R, E, N, K, dt, gather)
    ref, S = M.wgrad(X, dY, offsets, rows)
    for transb in "NT":
        dW = torch.full((E, K + 1, N + 3) if transb == "N" else (E, N + 1, K + 3), 9.0, dtype=dt, device="cuda")
        out = dW[:, :-1, 1:-2]
        emu.grouped_wgrad(X.cuda(), dY.cuda(), offsets.int().cuda(), dW=out, transb=transb, rows=_cuda(rows))
        M.check(out if transb == "N" else out.transpose(1, 2), ref, M.product_bar(ref, S, R, dt) + 16 * 2.0 ** -23 * S)
        assert (dW[:, -1] == 9).all() and (dW[:, :, 0] == 9).all() and (dW[:, :, -2:] == 9).all()


def test_one_matrix_for_all_experts(emu):
    """A broadcast matrix (stride 0): copied once."""
    X, W, offsets, _, _ = _case(8, 6000, 4, 1001, 1030, torch.bfloat16, False, 0.0)
    Y, S = M.grouped(X, W[:1].expand(4, -1, -1), offsets, None)
    got = emu.grouped_gemm(X.cuda(), W[:1].cuda().expand(4, -1, -1), offsets.int().cuda())
    M.check(got, Y, M.product_bar(Y, S, 1030, torch.bfloat16))


def test_wrong_offsets_in_pieces(emu):
    """Offsets out of order: each expert's rows as the product reads them."""
    gen = torch.Generator().manual_seed(3)
    X, dY = torch.randn((5000, 70), generator=gen), torch.randn((5000, 40), generator=gen)
    for offsets in ([-4, 2000, 1500, 2 ** 31 - 1], [7, 4000, 10, 5000]):
        got = emu.grouped_wgrad(X.cuda(), dY.cuda(), torch.tensor(offsets).int().cuda())
        for e in range(3):
            lo = min(max(offsets[e], 0), 5000) if e else 0
            hi = min(max(offsets[e + 1], lo), 5000)
            x, y = X[lo:hi].double(), dY[lo:hi].double()
            S = x.abs().T @ y.abs()
            M.check(got[e], x.T @ y, M.product_bar(x.T @ y, S, 5000, torch.float32) + 16 * 2.0 ** -23 * S)


def test_without_workspace(emu, monkeypatch):
    """Where the workspace may not grow, the same results without copies and pieces."""
    emu.release_workspace()
    monkeypatch.setenv("EMU_WORKSPACE_LIMIT", "4096")
    X, W, offsets, _, dY = _case(8, 5000, 2, 301, 1030, torch.bfloat16, False, 0.0)
    Y, S = M.grouped(X, W, offsets, None)
    M.check(emu.grouped_gemm(X.cuda(), W.cuda(), offsets.int().cuda()), Y, M.product_bar(Y, S, 1030, torch.bfloat16))
    ref, S = M.wgrad(X, dY, offsets, None)
    M.check(emu.grouped_wgrad(X.cuda(), dY.cuda(), offsets.int().cuda()), ref, M.product_bar(ref, S, 5000, torch.bfloat16))
    assert emu.workspace_bytes() <= 4096


def test_same_bits_every_time(emu):
    X, W, offsets, rows, dY = (_cuda(t) for t in _case(31, 5000, 3, 1001, 1030, torch.bfloat16, True))
    off = offsets.int()
    a, b = emu.grouped_gemm(X, W, off, rows=rows), emu.grouped_wgrad(X[:, :70], dY[:, :90], off, rows=rows)
    for _ in range(3):
        assert torch.equal(emu.grouped_gemm(X, W, off, rows=rows), a)
        assert torch.equal(emu.grouped_wgrad(X[:, :70], dY[:, :90], off, rows=rows), b)
