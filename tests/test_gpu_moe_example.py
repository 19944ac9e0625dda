"""The example's layer: its output and gradients against autograd in 64 bits, and the
4-bit form against the layer with the unpacked matrices."""
import importlib.util
import os

import pytest
import torch

import _moe as M

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


def _reference(x, Wr, W1, W2, k, scope, ids):
    """The layer in 64 bits with the given choice of experts."""
    logits = x @ Wr
    chosen = torch.gather(logits, 1, ids)
    if scope == "chosen":
        weights = torch.softmax(chosen, 1)
    else:
        weights = torch.gather(torch.softmax(logits, 1), 1, ids)
    y = torch.zeros_like(x)
    for j in range(k):
        h = torch.matmul(W1[ids[:, j]], x[:, :, None])[:, :, 0]
        z = torch.matmul(W2[ids[:, j]], torch.nn.functional.silu(h)[:, :, None])[:, :, 0]
        y = y + weights[:, j:j + 1] * z
    return y


@pytest.mark.parametrize("T,D,H,E,k,scope", [(1, 64, 96, 4, 2, "chosen"), (70, 96, 65, 8, 3, "all"),
                                             (300, 130, 128, 5, 2, "chosen")])
def test_layer_and_gradients(layer, T, D, H, E, k, scope):
    """float32.  Every sum of the chain has at most D + H + T k terms, each within
    2^-23 (terms / 8 + 8) of the sums of magnitudes; 12 such sums follow one another
    at most, and the magnitudes of a sum of n random terms are below 4 sqrt(n) times
    its norm's share of an entry: the bar, relative to the largest entry."""
    gen = torch.Generator().manual_seed(T)
    x = torch.randn((T, D), generator=gen)
    Wr = torch.randn((D, E), generator=gen) / D ** 0.5
    W1, W2 = torch.randn((E, H, D), generator=gen) / D ** 0.5, torch.randn((E, D, H), generator=gen) / H ** 0.5
    dy = torch.randn((T, D), generator=gen)
    got = [t.cuda().requires_grad_() for t in (x, Wr, W1, W2)]
    y = layer.moe(*got, k, scope)
    y.backward(dy.cuda())
    ids = torch.sort(x.double() @ Wr.double(), dim=1, descending=True, stable=True)[1][:, :k]
    ref = [t.double().requires_grad_() for t in (x, Wr, W1, W2)]
    y64 = _reference(*ref, k, scope, ids)
    y64.backward(dy.double())
    n = D + H + T * k
    bar = 12 * 2.0 ** -23 * (n / 8 + 8) * 4 * n ** 0.5
    for name, a, b in [("y", y.detach(), y64.detach())] + [
            (s, p.grad, q.grad) for s, p, q in zip(("x", "Wr", "W1", "W2"), got, ref)]:
        M.check(a, b, bar * b.abs().max() * torch.ones_like(b), name)


@pytest.mark.parametrize("tokens", [1, 5])
def test_served_from_4_bits(layer, tokens):
    """Against the layer in 64 bits with the matrices that the 4 bits stand for; the
    bar as above, all of it float32."""
    D, H, E, k = 128, 192, 6, 2
    gen = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, D), generator=gen)
    Wr = torch.randn((D, E), generator=gen) / D ** 0.5
    W1, W2 = torch.randn((E, H, D), generator=gen) / D ** 0.5, torch.randn((E, D, H), generator=gen) / H ** 0.5
    served = layer.Served(Wr.cuda(), W1.cuda(), W2.cuda(), k)
    got = served(x.cuda())
    back = [M.unpacked(q.cpu(), s.cpu(), None)[0] for q, s in (served.W1, served.W2)]
    ids = torch.sort(x.double() @ Wr.double(), dim=1, descending=True, stable=True)[1][:, :k]
    ref = _reference(x.double(), Wr.double(), *back, k, "chosen", ids)
    n = D + H
    M.check(got, ref, 12 * 2.0 ** -23 * (n / 8 + 55) * 4 * n ** 0.5 * ref.abs().max() * torch.ones_like(ref))


def test_the_example_runs(layer, capsys):
    assert layer.main(T=512, D=256, H=128, E=8, k=2, steps=6) < 1.2
    assert "4 bits" in capsys.readouterr().out
