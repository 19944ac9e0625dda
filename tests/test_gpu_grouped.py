"""Products grouped by expert and the gradient of the matrices against 64 bits."""
import math

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


def _case(seed, R, E, N, K, dt, gather, tail=0.1):
    """Uneven experts, some without rows; the last rows belong to none and hold NaN."""
    gen = torch.Generator().manual_seed(seed)
    live = R - int(tail * R)
    cuts = torch.sort(torch.randint(0, live + 1, (max(E - 1, 0),), generator=gen))[0]
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([live])))[-(E + 1):]
    offsets[0] = 0
    if E > 3:
        offsets[2] = offsets[1]                        # expert 1 has no rows
    if gather:
        T = max(1, R // 2)
        X = torch.randn((T, K), generator=gen).to(dt)
        rows = torch.randint(0, T, (R,), generator=gen).int()
        rows[live:] = -1
        if live > 2:
            rows[1] = T + 5                            # outside: a row of zeros
            rows[2] = -7
    else:
        X, rows = torch.randn((R, K), generator=gen).to(dt), None
        X[live:] = math.nan
    W = (torch.randn((E, K, N), generator=gen) / max(1, K) ** 0.5).to(dt)
    dY = torch.randn((R, N), generator=gen).to(dt)
    dY[live:] = math.nan
    return X, W, offsets, rows, dY


def _cuda(t):
    return None if t is None else t.cuda()


SHAPES = [  # R, E, N, K
    (1, 1, 1, 1), (1, 8, 64, 32), (2, 3, 130, 33), (33, 4, 17, 128), (100, 3, 129, 65),
    (128, 1, 128, 64), (129, 2, 256, 96), (300, 5, 250, 127), (513, 70, 96, 40), (700, 2, 385, 513),
    (1000, 130, 64, 72), (40, 2, 1, 200), (260, 1, 131, 1031)]


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K", SHAPES)
def test_product(emu, kind, R, E, N, K, transb, gather):
    dt = M.TYPES[kind]
    X, W, offsets, rows, _ = _case(R + N, R, E, N, K, dt, gather)
    Y, S = M.grouped(X, W, offsets, rows)
    w = W if transb == "N" else W.transpose(1, 2).contiguous()
    got = emu.grouped_gemm(X.cuda(), w.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    M.check(got, Y, M.product_bar(Y, S, K, dt))


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K", SHAPES)
def test_gradient_of_the_matrices(emu, kind, R, E, N, K, transb, gather):
    dt = M.TYPES[kind]
    X, _, offsets, rows, dY = _case(R + K, R, E, N, K, dt, gather)
    ref, S = M.wgrad(X, dY, offsets, rows)
    got = emu.grouped_wgrad(X.cuda(), dY.cuda(), offsets.int().cuda(), transb=transb, rows=_cuda(rows))
    if transb == "T":
        got = got.transpose(1, 2)
    M.check(got, ref, M.product_bar(ref, S, R, dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
def test_nothing_to_multiply(emu, kind):
    dt = M.TYPES[kind]
    off = torch.zeros(5, dtype=torch.int32, device="cuda")
    X, W = torch.ones((6, 40), dtype=dt, device="cuda"), torch.ones((4, 40, 70), dtype=dt, device="cuda")
    assert (emu.grouped_gemm(X, W, off) == 0).all()                       # no expert has rows
    assert emu.grouped_gemm(X[:0], W, off).shape == (0, 70)
    assert (emu.grouped_wgrad(X, torch.ones((6, 70), dtype=dt, device="cuda"), off) == 0).all()
    assert (emu.grouped_wgrad(X[:0], X[:0], off) == 0).all()
    off[1:] = 6
    assert (emu.grouped_gemm(X[:, :0], W[:, :0], off) == 0).all()          # K = 0


def test_offsets_that_are_wrong_stay_inside(emu):
    """Offsets are clamped to the rows that exist, a decreasing one to its expert's start."""
    gen = torch.Generator().manual_seed(2)
    X = torch.randn((50, 64), generator=gen)
    W = torch.randn((3, 64, 40), generator=gen)
    for offsets in ([-4, 20, 60, 2 ** 31 - 1], [7, 20, 30, 50], [0, 10, 10, 1000]):
        offsets = torch.tensor(offsets)
        Y, S = M.grouped(X, W, offsets, None)
        got = emu.grouped_gemm(X.cuda(), W.cuda(), offsets.int().cuda())
        M.check(got, Y, M.product_bar(Y, S, 64, torch.float32), str(offsets))


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("transb", ["N", "T"])
def test_strides_and_alignment(emu, kind, transb):
    """Operands and outputs inside larger matrices, at odd element offsets."""
    dt = M.TYPES[kind]
    R, E, N, K = 150, 3, 140, 99
    X, W, offsets, rows, dY = _case(12, R, E, N, K, dt, True)
    X[X != X] = 0
    big_x = torch.full((X.shape[0], K + 7), math.nan, dtype=dt)
    big_x[:, 5:5 + K] = X
    a, b = (K, N) if transb == "N" else (N, K)
    big_w = torch.full((E, a + 3, b + 9), math.nan, dtype=dt)
    big_w[:, 1:1 + a, 3:3 + b] = W if transb == "N" else W.transpose(1, 2)
    out = torch.full((R, N + 3), 9.0, dtype=dt, device="cuda")
    xc, wc, off = big_x.cuda()[:, 5:5 + K], big_w.cuda()[:, 1:1 + a, 3:3 + b], offsets.int().cuda()
    emu.grouped_gemm(xc, wc, off, Y=out[:, 1:1 + N], transb=transb, rows=rows.cuda())
    Y, S = M.grouped(X, W, offsets, rows)
    M.check(out[:, 1:1 + N], Y, M.product_bar(Y, S, K, dt))
    assert (out[:, 0] == 9).all() and (out[:, N + 1:] == 9).all()
    dw = torch.full((E, a + 1, b + 5), 9.0, dtype=dt, device="cuda")
    big_y = torch.full((R, N + 11), math.nan, dtype=dt)
    big_y[:, 7:7 + N] = dY
    emu.grouped_wgrad(xc, big_y.cuda()[:, 7:7 + N], off, dW=dw[:, :a, 3:3 + b], transb=transb,
                      rows=rows.cuda())
    ref, S = M.wgrad(X, dY, offsets, rows)
    got = dw[:, :a, 3:3 + b]
    M.check(got if transb == "N" else got.transpose(1, 2), ref, M.product_bar(ref, S, R, dt))
    assert (dw[:, a:] == 9).all() and (dw[:, :, :3] == 9).all() and (dw[:, :, 3 + b:] == 9).all()


def test_gradients_by_differences(emu):
    """The product is linear in X and in W: a step of one along a direction
    changes <Y, dY> by that direction's product with the gradient.  The bar is
    the products' own (2^-23 (K / 8 + 8) of the sums of magnitudes), for the
    two differences and the gradient."""
    R, E, N, K = 90, 4, 70, 50
    X, W, offsets, _, dY = (None if t is None else t for t in _case(4, R, E, N, K, torch.float32, False, 0.0))
    off = offsets.int().cuda()
    gen = torch.Generator().manual_seed(5)
    vX, vW = torch.randn(X.shape, generator=gen), torch.randn(W.shape, generator=gen)
    Xc, Wc, dYc = X.cuda(), W.cuda(), dY.cuda()
    dX = emu.grouped_gemm(dYc, Wc, off, transb="T")
    dW = emu.grouped_wgrad(Xc, dYc, off)

    def loss(X, W):
        return float((emu.grouped_gemm(X, W, off).double() * dYc.double()).sum())

    def magnitude(X, W):
        return float((M.grouped(X.abs(), W.abs(), offsets, None)[0] * dY.abs().double()).sum())

    bar = 2.0 ** -23 * (R / 8 + K / 8 + 16) * 3
    step = (loss(Xc + vX.cuda(), Wc) - loss(Xc - vX.cuda(), Wc)) / 2
    assert abs(step - float((dX.double() * vX.cuda()).sum())) <= bar * magnitude(X.abs() + vX.abs(), W)
    step = (loss(Xc, Wc + vW.cuda()) - loss(Xc, Wc - vW.cuda())) / 2
    assert abs(step - float((dW.double() * vW.cuda()).sum())) <= bar * magnitude(X, W.abs() + vW.abs())


def test_single_precision_keeps_small_terms(emu):
    """Exact integer products whose sums FP32 holds: every bit of the result."""
    gen = torch.Generator().manual_seed(6)
    X = torch.randint(-1000, 1001, (200, 16), generator=gen).float()
    W = torch.randint(-1000, 1001, (2, 16, 130), generator=gen).float()
    offsets = torch.tensor([0, 90, 200])
    Y, _ = M.grouped(X, W, offsets, None)
    got = emu.grouped_gemm(X.cuda(), W.cuda(), offsets.int().cuda())
    assert torch.equal(got.cpu().double(), Y)


def test_matrices_beyond_32_bit_offsets(emu):
    """The last expert's matrix starts past element 2^31."""
    E, N, K = 9, 16384, 16384
    W = torch.empty((E, N, K), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(7)
    W[-1] = torch.randn((N, K), generator=gen, device="cuda").to(torch.bfloat16)
    X = torch.randn((40, K), generator=gen, device="cuda").to(torch.bfloat16)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[-1] = 40
    got = emu.grouped_gemm(X, W, off, transb="T")
    cols = torch.tensor([0, 1, 5000, N - 1])
    ref = X.double().cpu() @ W[-1][cols.cuda()].double().cpu().T
    S = X.double().cpu().abs() @ W[-1][cols.cuda()].double().cpu().abs().T
    M.check(got[:, cols.cuda()], ref, M.product_bar(ref, S, K, torch.bfloat16))
    del W
    torch.cuda.empty_cache()


def test_same_bits_every_time(emu):
    for kind in M.TYPES:
        X, W, offsets, rows, dY = (_cuda(t) for t in _case(31, 600, 9, 200, 300, M.TYPES[kind], True))
        off = offsets.int()
        a, b = emu.grouped_gemm(X, W, off, rows=rows), emu.grouped_wgrad(X, dY, off, rows=rows)
        for _ in range(3):
            assert torch.equal(emu.grouped_gemm(X, W, off, rows=rows), a)
            assert torch.equal(emu.grouped_wgrad(X, dY, off, rows=rows), b)


def test_on_another_stream(emu):
    X, W, offsets, rows, _ = (_cuda(t) for t in _case(41, 500, 6, 300, 200, torch.float32, True))
    off = offsets.int()
    ref = emu.grouped_gemm(X, W, off, rows=rows)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Y = emu.grouped_gemm(X, W, off, rows=rows)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, ref)
    emu.lib().emu_set_stream(None)
