"""moe_route's results are tensors of their own (no kernel is launched)."""
import pytest
import torch

import paper_2609_04663_amd as emu


@pytest.fixture
def routing(monkeypatch):
    monkeypatch.setattr(emu, "_same_gpu", lambda *named: None)
    monkeypatch.setattr(emu, "_launch", lambda fn, device, *args: None)
    return emu.moe_route(torch.zeros((6, 9), dtype=torch.bfloat16), 3)


def test_shapes_and_types(routing):
    assert [tuple(t.shape) for t in routing] == [(6, 3), (6, 3), (10,), (18,), (6, 3)]
    assert [t.dtype for t in routing] == [torch.int32, torch.float32] + 3 * [torch.int32]
    assert all(t.is_contiguous() for t in routing)


def test_one_may_be_kept_without_the_others(routing):
    for t in routing:
        assert t.untyped_storage().nbytes() == t.numel() * t.element_size()
    assert len({t.untyped_storage().data_ptr() for t in routing}) == 5


def test_one_may_be_changed_while_autograd_holds_the_others(routing):
    class Holds(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            ctx.save_for_backward(routing.ids, routing.offsets, routing.rows, routing.slots)
            return x * 2

        @staticmethod
        def backward(ctx, dy):
            assert len(ctx.saved_tensors) == 4
            return dy * 2

    x = torch.ones(3, requires_grad=True)
    y = Holds.apply(x)
    routing.weights.mul_(0.5)
    y.sum().backward()
    assert (x.grad == 2).all()
