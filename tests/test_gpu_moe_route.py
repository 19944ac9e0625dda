"""The router against its definition: choices, order and offsets exactly, weights
and gradients within bars derived from their roundings."""
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


def _weight_bar(logits, weights):
    """exp's argument is off by 2^-24 of its size (at most the range of the
    logits), exp itself, the sum and the quotient by a few units."""
    x = logits.double()
    x = torch.where(torch.isfinite(x), x, 0.0)
    span = float(x.max() - x.min()) if x.numel() else 0.0
    return 2.0 ** -23 * (16 + span) * weights + 1e-37


def _check(emu, logits, k, scope):
    r = emu.moe_route(logits.cuda() if not logits.is_cuda else logits, k, scope)
    ref = M.route(logits.cpu(), k, scope)
    for name, got, want in (("ids", r.ids, ref[0]), ("offsets", r.offsets, ref[2]),
                            ("rows", r.rows, ref[3]), ("slots", r.slots, ref[4])):
        assert torch.equal(got.cpu().long(), want), name
    M.check(r.weights, ref[1], _weight_bar(logits.cpu(), ref[1]), "weights")
    return r, ref


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("T,E,k,scope", [
    (0, 8, 2, "all"), (1, 1, 1, "chosen"), (1, 64, 8, "all"), (5, 7, 7, "chosen"),
    (63, 64, 1, "all"), (64, 65, 3, "chosen"), (65, 128, 8, "all"), (200, 129, 17, "chosen"),
    (129, 256, 32, "all"), (70, 300, 5, "chosen"), (66, 1024, 32, "all"), (1500, 60, 4, "chosen")])
def test_route(emu, kind, T, E, k, scope):
    gen = torch.Generator().manual_seed(1000 * E + T)
    logits = (2 * torch.randn((T, E), generator=gen)).to(M.TYPES[kind])
    _check(emu, logits, k, scope)


@pytest.mark.parametrize("scope", ["chosen", "all"])
def test_ties_masks_and_values_that_are_not_numbers(emu, scope):
    gen = torch.Generator().manual_seed(3)
    x = torch.randint(-2, 3, (150, 33), generator=gen).float()      # many equal logits
    x[x == 0] *= torch.where(torch.rand(int((x == 0).sum()), generator=gen) < 0.5, -1.0, 1.0)  # -0 = 0
    x[3] = -math.inf                                                # no expert at all
    x[4] = -math.inf
    x[4, 9] = 1.0                                                   # one, of six asked for
    x[5, ::2] = math.nan
    x[6] = math.nan
    x[7] = torch.finfo(torch.float32).min                           # masks of the lowest value: all equal
    x[8] = torch.finfo(torch.float32).min
    x[8, 30] = 0.0
    x[9, 5] = x[9, 20] = math.inf                                   # the two share the weight
    x[10] = math.inf
    x[11, 1:] = -math.inf
    ref = x.clone()
    ref[torch.isnan(ref)] = -math.inf
    r = emu.moe_route(x.cuda(), 6, scope)
    ids, weights, offsets, rows, slots = M.route(ref, 6, scope)
    assert torch.equal(r.ids.cpu().long(), ids)
    assert torch.equal(r.offsets.cpu().long(), offsets)
    assert torch.equal(r.rows.cpu().long(), rows) and torch.equal(r.slots.cpu().long(), slots)
    M.check(r.weights, weights, 2.0 ** -23 * 24 * weights + 1e-37, "weights")


def test_rows_of_a_larger_matrix(emu):
    gen = torch.Generator().manual_seed(4)
    whole = torch.randn((300, 101), generator=gen).to(torch.bfloat16)
    part = whole[:, 3:67]
    ref = M.route(part, 4, "all")
    r = emu.moe_route(whole.cuda()[:, 3:67], 4, "all")
    assert torch.equal(r.ids.cpu().long(), ref[0]) and torch.equal(r.rows.cpu().long(), ref[3])


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("T,E,k,scope", [(1, 8, 8, "all"), (37, 64, 8, "chosen"), (100, 130, 20, "all"),
                                         (50, 700, 32, "all"), (33, 700, 9, "chosen")])
def test_gradient_by_the_formula(emu, kind, T, E, k, scope):
    gen = torch.Generator().manual_seed(E + T)
    dt = M.TYPES[kind]
    logits = torch.randn((T, E), generator=gen).to(dt)
    logits[torch.rand((T, E), generator=gen) < 0.2] = -math.inf
    logits[T // 2] = -math.inf
    dw = torch.randn((T, k), generator=gen)
    r = emu.moe_route(logits.cuda(), k, scope)
    dead = r.ids.cpu() < 0
    dw[dead] = math.nan                                 # never used
    got = emu.moe_route_grad(logits.cuda(), r.ids, r.weights, dw.cuda(), scope)
    dw[dead] = 0.0
    ref = M.route_grad(logits, r.ids.cpu(), dw, scope)
    # each weight is off by at most 32 units of 2^-23 (range below 16); the mean
    # adds k terms no larger than the largest |dw|; one rounding to the type
    size = dw.abs().amax(1, keepdim=True).double()
    weight = torch.zeros_like(ref)
    p = torch.softmax(logits.double().nan_to_num(neginf=-1e9), 1) if scope == "all" else torch.ones_like(ref)
    weight += p
    M.check(got, ref, 2.0 ** -22 * (32 + k) * size * weight + M.rounded(ref, dt), "dlogits")


@pytest.mark.parametrize("scope", ["chosen", "all"])
def test_gradient_by_differences(emu, scope):
    """Central differences of the weights themselves: with h = 2^-6 the third
    derivative of a softmax (at most 1) leaves h^2 / 6 of sum |dw|, the weights'
    roundings 2^-19 / (2 h)."""
    gen = torch.Generator().manual_seed(9)
    T, E, k, h = 12, 10, 4, 2.0 ** -6
    # logits apart by 0.25, so that a step does not change the choice
    logits = torch.stack([torch.randperm(E, generator=gen) for _ in range(T)]).float() * 0.25
    dw = torch.randn((T, k), generator=gen)
    r = emu.moe_route(logits.cuda(), k, scope)
    got = emu.moe_route_grad(logits.cuda(), r.ids, r.weights, dw.cuda(), scope).cpu()
    for e in range(E):
        step = torch.zeros_like(logits)
        step[:, e] = h
        up = emu.moe_route((logits + step).cuda(), k, scope)
        down = emu.moe_route((logits - step).cuda(), k, scope)
        assert torch.equal(up.ids, r.ids) and torch.equal(down.ids, r.ids)
        slope = ((up.weights - down.weights).cpu().double() * dw).sum(1) / (2 * h)
        bar = dw.abs().double().sum(1) * (h * h / 6 + 2.0 ** -19 / (2 * h)) + 1e-6
        assert ((got[:, e].double() - slope).abs() <= bar).all()
