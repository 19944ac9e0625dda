"""The router where its kernels change: counts added up by the order's workgroups or
by a kernel of their own, experts to a lane, and 16-bit logits packed with their index."""
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


def _reference(logits, k, scope):
    """ids, weights, offsets, rows, slots by a stable sort in 64 bits."""
    x = logits.double()
    T, E = x.shape
    value, ids = torch.sort(x, dim=1, descending=True, stable=True)
    value, ids = value[:, :k], ids[:, :k]
    there = value > -math.inf
    top = torch.where(there[:, :1], value[:, :1], 0.0)
    over = value if scope == "chosen" else x
    weights = torch.where(there, torch.exp(value - top) / torch.exp(over - top).sum(1, keepdim=True), 0.0)
    flat = torch.where(there, ids, E).reshape(-1)
    order = torch.argsort(flat, stable=True)
    slots = torch.empty_like(order)
    slots[order] = torch.arange(T * k)
    offsets = torch.searchsorted(flat[order], torch.arange(E + 1))
    rows = torch.where(flat[order] < E, order // k, -1)
    return torch.where(there, ids, -1), weights, offsets, rows, torch.where(there, slots.view(T, k), -1)


def _check(r, want):
    for name, value in zip(("ids", "offsets", "rows", "slots"), (want[0], *want[2:])):
        assert torch.equal(getattr(r, name).cpu().long(), value), name


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("T,E,k,scope", [
    (64, 257, 8, "all"), (65, 511, 32, "chosen"), (4096, 512, 8, "all"),     # 32 experts to a lane
    (4160, 512, 4, "all"), (2049, 513, 3, "chosen"),                          # counts at and past the bound
    (2100, 997, 2, "all"), (8200, 61, 6, "chosen"), (40000, 67, 2, "chosen")])
def test_shapes(emu, kind, T, E, k, scope):
    gen = torch.Generator().manual_seed(7 * E + T)
    # half of the logits lie on a coarse grid: many are equal
    x = 2 * torch.randn((T, E), generator=gen)
    x = torch.where(torch.rand((T, E), generator=gen) < 0.5, torch.round(x * 4) / 4, x)
    x[torch.rand(T, generator=gen) < 0.1] = -math.inf
    x[torch.rand((T, E), generator=gen) < 0.2] = -math.inf
    x = x.to(M.TYPES[kind])
    live = x.double()[x > -math.inf]
    # as for the other sizes: exp's argument to 2^-24 of the range, a few units more
    bar = 2.0 ** -23 * (16 + float(live.max() - live.min()))
    r, want = emu.moe_route(x.cuda(), k, scope), _reference(x, k, scope)
    _check(r, want)
    M.check(r.weights, want[1], bar * want[1] + 1e-37, "weights")


@pytest.mark.parametrize("E", [12, 200, 300, 700])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_all_bits_of_16_bit_logits(emu, kind, E):
    """Any bit pattern: subnormals, both zeros, infinities and NaN; neighbours stay apart."""
    gen = torch.Generator().manual_seed(E)
    bits = torch.randint(-(1 << 15), 1 << 15, (300, E), generator=gen).to(torch.int16)
    bits[:100] = (bits[:1, :1] + torch.randint(-3, 4, (100, E), generator=gen)).to(torch.int16)
    bits[100:120] = torch.randint(-4, 5, (20, E), generator=gen).to(torch.int16)
    bits[120:130] = torch.where(torch.rand((10, E), generator=gen) < 0.5, 0, -(1 << 15)).to(torch.int16)
    x = bits.view(M.TYPES[kind])
    ref = torch.where(torch.isnan(x), -math.inf, x)
    r = emu.moe_route(x.cuda(), 8, "chosen")
    _check(r, _reference(ref, 8, "chosen"))
    some = r.ids[:, 0].cpu() >= 0
    M.check(r.weights.sum(1)[some.cuda()], torch.ones(int(some.sum()), dtype=torch.float64),
            8 * 2.0 ** -23, "sum of the weights")
