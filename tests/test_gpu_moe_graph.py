"""A mixture-of-experts step captured in a HIP graph: every replay, with eager
work between, gives the eager result for the inputs of its time."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


@pytest.mark.parametrize("T", [4, 150])
def test_replays(emu, T):
    E, k, D = 16, 4, 256
    gen = torch.Generator(device="cuda").manual_seed(T)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    x, gate = normal(T, D), normal(T, E)
    W, Q, s = normal(E, D, D) / 16, *emu.q4_pack(normal(E, D, D) / 16, 64)

    def step():
        r = emu.moe_route(gate, k, "all")
        z = emu.grouped_gemm(x, W, r.offsets, rows=r.rows)
        z = emu.q4_gemm(z, Q, s, offsets=r.offsets)
        y = emu.moe_combine(z, r.slots, r.weights)
        dz, dw = emu.moe_combine_grad(x, z, r.slots, r.weights, r.rows)
        dW = emu.grouped_wgrad(x, dz, r.offsets, rows=r.rows)
        return y, dW, emu.moe_route_grad(gate, r.ids, r.weights, dw, "all"), r.rows, r.slots

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                       # grows the workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        x.copy_(normal(T, D))
        gate.copy_(normal(T, E))
        ref = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, ref):
            assert torch.equal(a, b), i
    emu.lib().emu_set_stream(None)
