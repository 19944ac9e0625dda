"""The grouped product with few rows of each expert: long reductions (X in several
chunks), blocks of 1 to 32 rows, experts that take most of the rows, against 64 bits."""
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


@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K,gather", [
    (16, 1, 66, 1500, False), (32, 1, 64, 2049, True), (31, 1, 130, 5000, False), (15, 2, 63, 4096, True),
    (30, 30, 33, 2300, True), (8, 1, 200, 8200, False), (7, 1, 65, 33000, False), (60, 20, 129, 31, True),
    (1, 1, 1, 40000, False)])
def test_product(emu, kind, R, E, N, K, gather, transb):
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = _case(R + N, R, E, N, K, dt, gather)
    Y, S = M.grouped(X, W, offsets, rows)
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(X.cuda(), w.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got, Y, M.product_bar(Y, S, K, dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("E", [9, 64, 200])
def test_all_rows_at_one_expert(emu, kind, E):
    """The choice of a kernel is by the average; one expert may have every row."""
    dt, R, N, K = M.TYPES[kind], 8 * E, 70, 96
    gen = torch.Generator().manual_seed(E)
    X = torch.randn((R, K), generator=gen).to(dt)
    W = (torch.randn((E, K, N), generator=gen) / 10).to(dt)
    offsets = torch.zeros(E + 1, dtype=torch.int64)
    offsets[E // 2:] = R
    Y, S = M.grouped(X, W, offsets, None)
    M.check(emu.grouped_gemm(X.cuda(), W.cuda(), offsets.int().cuda()), Y, M.product_bar(Y, S, K, dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
def test_an_infinite_entry_stays_in_its_row_and_column(emu, kind):
    """X[1, 5] = inf spoils row 1, W[0][:, 3] = NaN column 3 of its expert, nothing else;
    entries behind the last index and rows behind the last are not read."""
    dt, N, K = M.TYPES[kind], 67, 45
    X, W, offsets, rows, _ = _case(3, 12, 2, N, K, dt, False, 0.0)
    offsets = torch.tensor([0, 5, 12])
    Y, S = M.grouped(X, W, offsets, None)
    X[1, 5], W[0, :, 3] = float("inf"), float("nan")
    wide = torch.full((2, K + 3, N + 2), float("nan"), dtype=dt)
    wide[:, :K, :N] = W
    got = emu.grouped_gemm(X.cuda(), wide.cuda()[:, :K, :N], offsets.int().cuda()).cpu()
    spoiled = torch.zeros(got.shape, dtype=torch.bool)
    spoiled[1], spoiled[:5, 3] = True, True
    assert (~torch.isfinite(got[spoiled].float())).all()
    got[spoiled], Y[spoiled], S[spoiled] = 0, 0, 0
    M.check(got, Y, M.product_bar(Y, S, K, dt))


@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K", [(8, 1, 17000, 70), (30, 4, 4111, 100), (60, 2, 8200, 65), (400, 60, 1000, 64)])
def test_enough_columns_to_fill_the_chip(emu, kind, R, E, N, K, transb):
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = _case(R + N, R, E, N, K, dt, True)
    Y, S = M.grouped(X, W, offsets, rows)
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(X.cuda(), w.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got, Y, M.product_bar(Y, S, K, dt))
