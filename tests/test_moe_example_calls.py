"""Which operators the example's layer calls: the losses' only where they are asked for, the
experts' products in the backward pass only where y has a gradient (operators stood in for on
the CPU: results of the right shapes, and a log)."""
import importlib.util
import os

import pytest
import torch

PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "moe_layer.py")
T, D, H, E, k = 6, 4, 5, 3, 2


@pytest.fixture
def calls(monkeypatch):
    spec = importlib.util.spec_from_file_location("moe_layer", PATH)
    layer = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(layer)
    emu, log = layer.emu, []

    def stand_in(name, result):
        monkeypatch.setattr(emu, name, lambda *a, **kw: (log.append(name), result(*a, **kw))[1])

    ints = lambda *s: torch.zeros(s, dtype=torch.int32)                             # noqa: E731
    stand_in("sgemm", lambda A, B: A @ B)
    stand_in("sgemm_ex", lambda A, B, transa="N", transb="N": (A.T if transa == "T" else A) @ (
        B.T if transb == "T" else B))
    stand_in("moe_route", lambda x, k, scope: emu.Routing(ints(T, k), torch.ones(T, k), ints(E + 1), ints(T * k),
                                                          ints(T, k)))
    stand_in("moe_route_grad", lambda logits, *a: torch.ones_like(logits))
    stand_in("grouped_gemm", lambda X, W, o, transb="N", rows=None: torch.ones(
        T * k, W.shape[1] if transb == "T" else W.shape[2]))
    stand_in("grouped_wgrad", lambda X, dY, o, transb, rows=None: torch.ones(E, dY.shape[1], X.shape[1]))
    stand_in("moe_combine", lambda Z, slots, weights=None: torch.ones(T, Z.shape[1]))
    stand_in("moe_combine_grad", lambda dY, Z, s, w, rows: (torch.ones_like(Z), torch.ones_like(w)))
    stand_in("moe_balance", lambda x, ids: emu.Balance(torch.ones(1), torch.ones(1), ints(1, E), ints(1)))
    stand_in("moe_balance_grad", lambda logits, *a: torch.full_like(logits, 2))
    return layer, log


def _args():
    return [torch.ones(s).requires_grad_() for s in ((T, D), (D, E), (E, H, D), (E, D, H))]


def test_the_layer_alone_computes_no_loss(calls):
    layer, log = calls
    args = _args()
    y = layer.moe(*args, k)
    assert "moe_balance" not in log
    y.sum().backward()
    assert "moe_balance" not in log and "moe_balance_grad" not in log
    assert log.count("grouped_gemm") == 4 and log.count("grouped_wgrad") == 2
    assert all(a.grad.shape == a.shape for a in args)
    with torch.no_grad():
        layer.moe(*args, k, "all")
    assert "moe_balance" not in log


def test_losses_alone_run_no_expert_backwards(calls):
    layer, log = calls
    args = _args()
    _, loss, zloss = layer.moe_with_losses(*args, k)
    assert log.count("moe_balance") == 1
    del log[:]
    (loss + zloss).sum().backward()
    assert sorted(log) == ["moe_balance_grad", "sgemm_ex", "sgemm_ex"]
    assert (args[0].grad == 2 * E).all() and (args[1].grad == 2 * T).all()
    assert all(a.grad.shape == a.shape and (a.grad == 0).all() for a in args[2:])


def test_all_of_them(calls):
    layer, log = calls
    args = _args()
    y, loss, _ = layer.moe_with_losses(*args, k)
    del log[:]
    (y.sum() + loss.sum()).backward()
    assert [log.count(n) for n in ("moe_balance_grad", "moe_route_grad", "grouped_gemm", "grouped_wgrad")] == [1, 1, 2, 2]
    assert (args[1].grad == 3 * T).all()
