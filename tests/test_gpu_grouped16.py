"""The kernels of 16-bit operands that are copied straight to LDS (whole 16-byte
chunks): extents around their tiles of 128 and 256 and their k-blocks of 32,
against 64 bits."""
import pytest
import torch

import _moe as M
from test_gpu_grouped import _case, _cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("R,E,N,K", [
    (33, 1, 8, 32), (129, 1, 128, 64), (300, 4, 256, 96), (700, 20, 520, 128), (600, 1, 264, 64),
    (1100, 2, 512, 160), (1030, 2, 1000, 416), (2500, 3, 136, 32), (2600, 5, 257 * 8, 192)])
def test_product(emu, kind, R, E, N, K, transb, gather):
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = _case(R + N, R, E, N, K, dt, gather)
    Y, S = M.grouped(X, W, offsets, rows)
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(X.cuda(), w.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got, Y, M.product_bar(Y, S, K, dt))


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("R,E,N,K", [
    (1, 1, 8, 8), (31, 2, 128, 64), (33, 1, 256, 256), (400, 5, 264, 136), (130, 1, 520, 512),
    (900, 3, 512, 1032), (700, 40, 512, 520), (96, 1, 1000, 640)])
def test_gradient_of_the_matrices(emu, kind, R, E, N, K, transb, gather):
    dt = M.TYPES[kind]
    X, _, offsets, rows, dY = _case(R + K, R, E, N, K, dt, gather)
    ref, S = M.wgrad(X, dY, offsets, rows)
    got = emu.grouped_wgrad(X.cuda(), dY.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    if transb == "T":
        got = got.transpose(1, 2)
    M.check(got, ref, M.product_bar(ref, S, R, dt))


@pytest.mark.parametrize("transb", ["N", "T"])
def test_strides_of_whole_chunks(emu, transb):
    """Operands inside larger matrices whose rows still start on 16 bytes."""
    dt, R, E, N, K = torch.bfloat16, 700, 2, 264, 96
    X, W, offsets, rows, dY = _case(12, R, E, N, K, dt, True)
    big_x = torch.full((X.shape[0], K + 24), float("nan"), dtype=dt)
    big_x[:, 8:8 + K] = X
    a, b = (K, N) if transb == "N" else (N, K)
    big_w = torch.full((E, a + 3, b + 16), float("nan"), dtype=dt)
    big_w[:, 1:1 + a, 8:8 + b] = W if transb == "N" else W.transpose(1, 2)
    out = torch.full((R, N + 3), 9.0, dtype=dt, device="cuda")
    xc, wc, off = big_x.cuda()[:, 8:8 + K], big_w.cuda()[:, 1:1 + a, 8:8 + b], offsets.int().cuda()
    emu.grouped_gemm(xc, wc, off, Y=out[:, 1:1 + N], transb=transb, rows=rows.cuda())
    Y, S = M.grouped(X, W, offsets, rows)
    M.check(out[:, 1:1 + N], Y, M.product_bar(Y, S, K, dt))
    assert (out[:, 0] == 9).all() and (out[:, N + 1:] == 9).all()
    big_y = torch.full((R, N + 8), float("nan"), dtype=dt)
    big_y[:, 8:] = dY
    dw = torch.full((E, a + 1, b + 5), 9.0, dtype=dt, device="cuda")
    emu.grouped_wgrad(xc, big_y.cuda()[:, 8:], off, dW=dw[:, :a, 3:3 + b], transb=transb, rows=rows.cuda())
    ref, S = M.wgrad(X, dY, offsets, rows)
    got = dw[:, :a, 3:3 + b]
    M.check(got if transb == "N" else got.transpose(1, 2), ref, M.product_bar(ref, S, R, dt))
    assert (dw[:, a:] == 9).all() and (dw[:, :, :3] == 9).all() and (dw[:, :, 3 + b:] == 9).all()
