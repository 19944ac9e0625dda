"""The FP32 kernels on tiles of 256, 192 and 128 rows: extents around them, and
sizes at which each height is the one with the fewest rounds, against 64 bits."""
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
@pytest.mark.parametrize("R,E,N,K", [
    (64, 1, 128, 32), (129, 1, 130, 31), (257, 1, 127, 64), (400, 3, 300, 97), (2000, 8, 140, 33),
    (8192, 1, 1000, 20), (7000, 2, 1024, 24), (4100, 1, 2050, 40), (9000, 1, 1030, 8)])
def test_product(emu, R, E, N, K, transb, gather):
    X, W, offsets, rows, _ = _case(R + N, R, E, N, K, torch.float32, gather)
    Y, S = M.grouped(X, W, offsets, rows)
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(X.cuda(), w.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got, Y, M.product_bar(Y, S, K, torch.float32))


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("R,E,N,K", [
    (33, 1, 129, 257), (65, 4, 300, 191), (31, 3, 1000, 1500), (10, 8, 1030, 700), (40, 1, 4100, 2050)])
def test_gradient_of_the_matrices(emu, R, E, N, K, transb, gather):
    X, _, offsets, rows, dY = _case(R + K, R, E, N, K, torch.float32, gather)
    ref, S = M.wgrad(X, dY, offsets, rows)
    got = emu.grouped_wgrad(X.cuda(), dY.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    if transb == "T":
        got = got.transpose(1, 2)
    M.check(got, ref, M.product_bar(ref, S, R, torch.float32))
