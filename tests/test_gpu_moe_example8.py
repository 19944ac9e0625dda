"""The example's losses and their gradients against autograd in 64 bits, and its 8-bit
form against the layer with what the 8 bits stand for."""
import importlib.util
import os

import pytest
import torch

import _moe as M
import _q8 as Q

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "moe_layer.py")


@pytest.fixture(scope="module")
def layer():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("moe_layer", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("T,D,H,E,k", [(70, 96, 65, 8, 3), (300, 130, 128, 5, 2)])
def test_losses_and_gradients(layer, T, D, H, E, k):
    """The losses alone, then with y: gradients of x and Wr through the logits.  The logits
    are sums of D products in 32 bits, off by 2^-23 (D / 8 + 8) of a sum of magnitudes of
    about sqrt(D) entries of size one, 12 units; their gradients pass through two more
    sums of at most T products: the bar, relative to the largest entry."""
    gen = torch.Generator().manual_seed(T)
    x = torch.randn((T, D), generator=gen)
    Wr = torch.randn((D, E), generator=gen) / D ** 0.5
    W1, W2 = torch.randn((E, H, D), generator=gen) / D ** 0.5, torch.randn((E, D, H), generator=gen) / H ** 0.5
    got = [t.cuda().requires_grad_() for t in (x, Wr, W1, W2)]
    _, loss, zloss = layer.moe_with_losses(*got, k)
    (0.7 * loss.sum() + 0.3 * zloss.sum()).backward()
    a, b = (t.double().requires_grad_() for t in (x, Wr))
    logits = a @ b
    ids = torch.sort(logits.detach(), dim=1, descending=True, stable=True)[1][:, :k]
    f = torch.bincount(ids.reshape(-1), minlength=E).double() / (T * k)
    ref_loss = E * (f * torch.softmax(logits, 1).mean(0)).sum()
    ref_z = (torch.logsumexp(logits, 1) ** 2).mean()
    (0.7 * ref_loss + 0.3 * ref_z).backward()
    n = D + T
    bar = 4 * 2.0 ** -23 * (n / 8 + 8) * 4 * n ** 0.5
    for name, u, v in (("loss", loss[0], ref_loss), ("zloss", zloss[0], ref_z), ("x", got[0].grad, a.grad),
                       ("Wr", got[1].grad, b.grad)):
        v = v.detach()
        M.check(u, v, bar * v.abs().max() * torch.ones_like(v), name)
    assert (got[2].grad == 0).all() and (got[3].grad == 0).all()


def test_served_from_8_bits(layer):
    """Each product against its own plain form on what the layer packed."""
    T, D, H, E, k = 90, 128, 200, 6, 2
    gen = torch.Generator().manual_seed(2)
    x = torch.randn((T, D), generator=gen)
    Wr = torch.randn((D, E), generator=gen) / D ** 0.5
    W1, W2 = torch.randn((E, H, D), generator=gen) / D ** 0.5, torch.randn((E, D, H), generator=gen) / H ** 0.5
    served = layer.Served8(Wr.cuda(), W1.cuda(), W2.cuda(), k)
    for got, w in ((served.W1, W1), (served.W2, W2)):
        q, s = Q.pack(w)
        assert torch.equal(got[0].cpu(), q) and torch.equal(got[1].cpu(), s)
    exact = layer.moe(x.cuda(), Wr.cuda(), W1.cuda(), W2.cuda(), k)
    # four packings, each off by at most half a 127th of a row's largest entry: below 1.5 % of its
    # norm where the largest is at most 4 times a typical entry (2 / 127 / sqrt(12) 4 < 0.9 %), the
    # products' errors add at random, and an activation's slope is below 1.1
    off = served(x.cuda()) - exact
    assert float(off.norm() / exact.norm()) < 0.06


def test_the_example_says_so(layer, capsys):
    layer.main(T=256, D=128, H=64, E=4, k=2, steps=2)
    assert "8 bits" in capsys.readouterr().out
