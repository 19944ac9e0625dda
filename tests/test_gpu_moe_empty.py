"""Products with an X without rows: every row number stands for a row of zeros."""
import pytest
import torch

import _moe as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


def _index(R):
    rows = torch.full((R,), -1, dtype=torch.int32)
    rows[::3], rows[1::3] = 0, 2 ** 31 - 1
    return rows.cuda()


@pytest.mark.parametrize("K", [192, 70])
@pytest.mark.parametrize("R", [5, 40, 1500])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", list(M.TYPES))
def test_products(emu, kind, transb, R, K):
    dt, E, N = M.TYPES[kind], 3, 130
    X = torch.empty((0, K), dtype=dt, device="cuda")
    W = torch.ones((E, K, N) if transb == "N" else (E, N, K), dtype=dt, device="cuda")
    off = torch.tensor([0, R // 2, R // 2, R], dtype=torch.int32, device="cuda")
    Y = torch.full((R, N), 9.0, dtype=dt, device="cuda")
    assert (emu.grouped_gemm(X, W, off, Y=Y, transb=transb, rows=_index(R)) == 0).all()
    dW = torch.full(W.shape, 9.0, dtype=dt, device="cuda")
    dY = torch.ones((R, N), dtype=dt, device="cuda")
    assert (emu.grouped_wgrad(X, dY, off, dW=dW, transb=transb, rows=_index(R)) == 0).all()


@pytest.mark.parametrize("R", [1, 7, 40, 300])
@pytest.mark.parametrize("kind", list(M.TYPES))
def test_4_bits(emu, kind, R):
    dt, N, K = M.TYPES[kind], 50, 256
    X = torch.empty((0, K), dtype=dt, device="cuda")
    Q = torch.zeros((2, N, K // 2), dtype=torch.uint8, device="cuda")
    s = torch.ones((2, N, K // 64), dtype=dt, device="cuda")
    off = torch.tensor([0, R // 2, R], dtype=torch.int32, device="cuda")
    Y = torch.full((R, N), 9.0, dtype=dt, device="cuda")
    assert (emu.q4_gemm(X, Q, s, offsets=off, rows=_index(R), Y=Y) == 0).all()


@pytest.mark.parametrize("kind", list(M.TYPES))
def test_some_rows_outside(emu, kind):
    """Rows outside next to rows that are there, in long and short reductions."""
    for R, K in ((700, 200), (300, 33), (200, 1000)):
        dt, E, N = M.TYPES[kind], 2, 96
        gen = torch.Generator().manual_seed(K)
        X, W = torch.randn((50, K), generator=gen).to(dt), (torch.randn((E, K, N), generator=gen) / 8).to(dt)
        rows = torch.randint(-20, 70, (R,), generator=gen).int()
        off = torch.tensor([0, R // 3, R])
        for transb in "NT":
            w = W if transb == "N" else W.transpose(1, 2).contiguous()
            Y, S = M.grouped(X, W, off, rows)
            got = emu.grouped_gemm(X.cuda(), w.cuda(), off.int().cuda(), transb=transb, rows=rows.cuda())
            M.check(got, Y, M.product_bar(Y, S, K, dt))


def test_by_the_c_entry_points(emu):
    """The same with a pointer that is not NULL, at the end of an allocation."""
    L, K, N, R = emu.lib(), 4096, 64, 300
    guard = torch.ones(K, device="cuda")
    W, Y = torch.ones((1, N, K), device="cuda"), torch.full((R, N), 9.0, device="cuda")
    off, rows = torch.tensor([0, R], dtype=torch.int32, device="cuda"), _index(R)
    emu._bind_stream(torch.device("cuda", 0))
    rc = L.emu_grouped_gemm(0, b"T", 1, R, N, K, guard.data_ptr(), K, 0, rows.data_ptr(), W.data_ptr(), K, N * K,
                            off.data_ptr(), Y.data_ptr(), N)
    assert rc == emu.EMU_OK and (Y == 0).all()


@pytest.mark.parametrize("R", [3, 9000])
@pytest.mark.parametrize("kind", list(M.TYPES))
def test_gradient_of_the_combination_without_tokens(emu, kind, R):
    """A buffer of rows that no token uses: their gradient is zero."""
    dt, D, k = M.TYPES[kind], 70, 2
    Z = torch.full((R, D), float("nan"), dtype=dt, device="cuda")
    dZ, dw = emu.moe_combine_grad(Z[:0], Z, torch.empty((0, k), dtype=torch.int32, device="cuda"),
                                  torch.empty((0, k), device="cuda"), torch.full((R,), -1, dtype=torch.int32, device="cuda"))
    assert dZ.shape == (R, D) and (dZ == 0).all() and dw.shape == (0, k)
