"""The weighted sum of the experts' rows and its gradients against 64 bits."""
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


def _case(seed, T, D, k, dt, dead=0.2):
    gen = torch.Generator().manual_seed(seed)
    Z = torch.randn((T * k, D), generator=gen).to(dt)
    w = torch.randn((T, k), generator=gen)
    alive = torch.rand(T * k, generator=gen) >= dead
    order = torch.cat((torch.nonzero(alive)[:, 0][torch.randperm(int(alive.sum()), generator=gen)],
                       torch.nonzero(~alive)[:, 0]))
    slots = torch.empty(T * k, dtype=torch.int64)
    slots[order] = torch.arange(T * k)
    slots[~alive] = -1
    rows = torch.where(alive[order], order // k, -1)
    slots = slots.view(T, k)
    # what belongs to no token may hold anything
    Z[rows < 0] = math.nan
    w[slots < 0] = math.nan
    return Z, w, slots.int(), rows.int()


def _reference(Z, w, slots):
    T, k = slots.shape
    Y = torch.zeros((T, Z.shape[1]), dtype=torch.float64)
    S = torch.zeros_like(Y)
    for t in range(T):
        for j in range(k):
            if slots[t, j] >= 0:
                term = float(w[t, j]) * Z[int(slots[t, j])].double()
                Y[t] += term
                S[t] += term.abs()
    return Y, S


SHAPES = [(1, 1, 1), (1, 4096, 8), (3, 7, 2), (17, 64, 5), (40, 1001, 8), (9, 2051, 32), (130, 256, 3)]


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("T,D,k", SHAPES)
def test_sum(emu, kind, T, D, k):
    dt = M.TYPES[kind]
    Z, w, slots, _ = _case(T + D, T, D, k, dt)
    Y, S = _reference(Z, w, slots)
    # k fused multiply-adds in 32 bits, one rounding to the type
    M.check(emu.moe_combine(Z.cuda(), slots.cuda(), w.cuda()), Y, 2.0 ** -24 * k * S + M.rounded(Y, dt))
    ones = torch.ones_like(w)
    Y, S = _reference(Z, ones, slots)
    M.check(emu.moe_combine(Z.cuda(), slots.cuda()), Y, 2.0 ** -24 * k * S + M.rounded(Y, dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("T,D,k", SHAPES)
def test_gradients(emu, kind, T, D, k):
    dt = M.TYPES[kind]
    Z, w, slots, rows = _case(3 * T + D, T, D, k, dt)
    dY = torch.randn((T, D), generator=torch.Generator().manual_seed(D)).to(dt)
    dZ, dw = emu.moe_combine_grad(dY.cuda(), Z.cuda(), slots.cuda(), w.cuda(), rows.cuda())
    ref_z = torch.zeros(Z.shape, dtype=torch.float64)
    ref_w = torch.zeros(w.shape, dtype=torch.float64)
    S = torch.zeros_like(ref_w)
    for t in range(T):
        for j in range(k):
            at = int(slots[t, j])
            if at >= 0:
                ref_z[at] = float(w[t, j]) * dY[t].double()
                ref_w[t, j] = (Z[at].double() * dY[t].double()).sum()
                S[t, j] = (Z[at].double() * dY[t].double()).abs().sum()
    # one product in 32 bits and its rounding to the type
    M.check(dZ, ref_z, 2.0 ** -24 * ref_z.abs() + M.rounded(ref_z, dt), "dZ")
    # a lane adds at most D / 64 + 8 products, ten more sums join the lanes
    M.check(dw, ref_w, 2.0 ** -24 * (D / 64 + 20) * S + 1e-37, "dweights")


def test_gradients_by_differences(emu):
    """The sum is linear in Z and in the weights, so a step of one along any
    direction changes <Y, dY> by that direction's product with the gradient, but
    for the roundings: of about 2 x 2^-24 x terms x their size."""
    Z, w, slots, rows = (t.cuda() for t in _case(5, 25, 130, 4, torch.float32, dead=0.0))
    gen = torch.Generator().manual_seed(6)
    dY, vZ, vw = (torch.randn(s, generator=gen).cuda() for s in ((25, 130), Z.shape, w.shape))
    dZ, dw = emu.moe_combine_grad(dY, Z, slots, w, rows)

    def loss(Z, w):
        return (emu.moe_combine(Z, slots, w).double() * dY.double()).sum()

    terms = float((Z.abs().double().sum() + vZ.abs().double().sum()) * 8 * 4)
    bar = 2.0 ** -22 * terms
    assert abs(float((loss(Z + vZ, w) - loss(Z - vZ, w)) / 2 - (dZ.double() * vZ).sum())) <= bar
    assert abs(float((loss(Z, w + vw) - loss(Z, w - vw)) / 2 - (dw.double() * vw).sum())) <= bar


def test_strides_and_outputs(emu):
    gen = torch.Generator().manual_seed(8)
    T, D, k = 21, 37, 3
    Z, w, slots, rows = _case(7, T, D, k, torch.float16)
    Y, S = _reference(Z, w, slots)
    big = torch.full((T * k, D + 9), 5.0, dtype=torch.float16)
    big[:, 3:3 + D] = Z
    out = torch.full((T, D + 5), 7.0, dtype=torch.float16, device="cuda")
    emu.moe_combine(big.cuda()[:, 3:3 + D], slots.cuda(), w.cuda(), Y=out[:, 1:1 + D])
    M.check(out[:, 1:1 + D], Y, 2.0 ** -24 * k * S + M.rounded(Y, torch.float16))
    assert (out[:, 0] == 7).all() and (out[:, 1 + D:] == 7).all()
    wide = torch.randn((T, 2 * D), generator=gen).to(torch.float16)
    dZ, _ = emu.moe_combine_grad(wide.cuda()[:, D:], big.cuda()[:, 3:3 + D], slots.cuda(), w.cuda(),
                                 rows.cuda())
    for t in range(T):
        for j in range(k):
            if slots[t, j] >= 0:
                ref = float(w[t, j]) * wide[t, D:].double()
                assert ((dZ[int(slots[t, j])].cpu().double() - ref).abs()
                        <= 2.0 ** -24 * ref.abs() + M.rounded(ref, torch.float16)).all()


def test_slots_outside_and_no_rows(emu):
    Z = torch.ones((4, 16), device="cuda")
    slots = torch.tensor([[0, 4], [-5, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    Y = emu.moe_combine(Z, slots, torch.ones((2, 2), device="cuda"))
    assert (Y[0] == 1).all() and (Y[1] == 0).all()
    Y = emu.moe_combine(Z[:0], slots, torch.ones((2, 2), device="cuda"))
    assert (Y == 0).all()
    assert emu.moe_combine(Z, slots[:0], torch.ones((0, 2), device="cuda")).shape == (0, 16)


def test_rows_beyond_32_bit_offsets(emu):
    """Row 2^20 + 7 of 4096 entries starts past element 2^32."""
    D = 4096
    Z = torch.empty((2 ** 20 + 8, D), dtype=torch.float16, device="cuda")
    Z[-1] = torch.arange(D, device="cuda").half() / 64
    slots = torch.tensor([[2 ** 20 + 7]], dtype=torch.int32, device="cuda")
    w = torch.full((1, 1), 0.5, device="cuda")
    assert torch.equal(emu.moe_combine(Z, slots, w)[0], Z[-1] / 2)
    del Z
    torch.cuda.empty_cache()
