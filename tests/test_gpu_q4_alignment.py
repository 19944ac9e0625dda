"""4-bit matrices, scales and offsets that start at any of their elements."""
import pytest
import torch

import _moe as M
from test_gpu_q4 import _bar, _matrices, _reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


def _at(t, first):
    """t, contiguous, from element `first` of an allocation."""
    room = torch.empty(t.numel() + first, dtype=t.dtype, device="cuda")
    part = room[first:].view(t.shape)
    part.copy_(t)
    return part


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R", [1, 9, 20, 70])
def test_any_element(emu, kind, R):
    dt, N, K, group = M.TYPES[kind], 70, 640, 32
    gen = torch.Generator().manual_seed(R)
    X = torch.randn((R, K), generator=gen).to(dt)
    Q, s, m = _matrices(gen, 1, N, K, group, dt, True)
    Y, S = _reference(X, Q, s, m, torch.tensor([0, R]), None)
    for q, f in ((1, 1), (2, 3), (3, 0), (6, 5)):
        got = emu.q4_gemm(X.cuda(), _at(Q, q), _at(s, f), mins=_at(m, f))
        M.check(got, Y, _bar(Y, S, K, group, dt))
    W = torch.randn((6, 96), generator=gen).to(dt)
    whole, scales = emu.q4_pack(W.cuda(), 32)
    part, part_scales = emu.q4_pack(_at(W, 1), 32)
    assert torch.equal(whole, part) and torch.equal(scales, part_scales)
