"""Operators that use the workspace for copies, pieces and split sums, in one captured
graph: every replay gives the eager bits."""
import pytest
import torch

import _moe_shapes as S
from test_gpu_grouped import _case, _cuda

pytestmark = pytest.mark.gpu


def test_replays():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as emu
    emu.lib()
    X, W, off, _, _ = (_cuda(t) for t in _case(1, *S.COPIED, torch.bfloat16, False, 0.0))
    R, E, N, K = S.PIECES
    x, _, at, _, dy = (_cuda(t) for t in _case(2, R, E, N, K, torch.float32, False, 0.0))
    R4, _, N4, K4, group = S.SPLIT
    gen = torch.Generator(device="cuda").manual_seed(3)
    x4 = torch.randn((R4, K4), generator=gen, device="cuda")
    Q = torch.randint(0, 256, (1, N4, K4 // 2), generator=gen, device="cuda", dtype=torch.uint8)
    s = torch.rand((1, N4, K4 // group), generator=gen, device="cuda")
    off, at = off.int(), at.int()

    def step():
        return emu.grouped_gemm(X, W, off), emu.grouped_wgrad(x, dy, at), emu.q4_gemm(x4, Q, s)

    step()                                              # grows the workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        for t in (X, x, x4):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        want = [t.clone() for t in step()]
        for t in captured:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b), i
    emu.lib().emu_set_stream(None)
