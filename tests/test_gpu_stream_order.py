"""Graphs whose branches share the workspace, and calls outside before and after a
capture: every replay gives the bits of the calls alone."""
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


def _calls(emu, seed):
    """Two calls that use the workspace (split planes; 4-bit sums in parts), as functions
    of their outputs, with inputs that can be refreshed."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    A, B = (torch.randn((1024, 1024), generator=gen, device="cuda") for _ in range(2))
    X = torch.randn((5, 16384), generator=gen, device="cuda")
    Q = torch.randint(0, 256, (1, 64, 8192), generator=gen, device="cuda", dtype=torch.uint8)
    s = torch.rand((1, 64, 256), generator=gen, device="cuda")
    return (lambda: emu.sgemm(A, B)), (lambda: emu.q4_gemm(X, Q, s)), (A, X)


def test_branches_of_a_graph(emu):
    one, two, inputs = _calls(emu, 1)
    one(), two()                                     # grows the workspace
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        a = one()
        with torch.cuda.stream(side):
            b = two()
        c = one()
        main.wait_stream(side)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for i in range(5):
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        want = [one().clone(), two().clone()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and torch.equal(c, want[0]), i
    emu.lib().emu_set_stream(None)


def test_calls_before_and_after_a_capture(emu):
    """Work on one stream, a capture on another, work on a third: in that order."""
    one, two, _ = _calls(emu, 3)
    want = [one().clone(), two().clone()]
    torch.cuda.synchronize()
    s0, s1, s2 = (torch.cuda.Stream() for _ in range(3))
    for _ in range(3):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s0):
            got = [one() for _ in range(4)]
        with torch.cuda.stream(s1):
            graph.capture_begin(capture_error_mode="thread_local")
            inside = two()
            graph.capture_end()
        with torch.cuda.stream(s2):
            after = two()
        torch.cuda.synchronize()
        assert all(torch.equal(g, want[0]) for g in got) and torch.equal(after, want[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(inside, want[1])
    emu.lib().emu_set_stream(None)


def test_a_graph_after_the_workspace_has_grown(emu):
    """Larger calls, and others' allocations, after the capture."""
    one, two, inputs = _calls(emu, 4)
    emu.release_workspace()
    one(), two()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = one(), two()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for n in (1024, 3000, 5000):
        A = torch.randn((n, n), generator=gen, device="cuda")
        emu.sgemm(A, A)
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        want = [one().clone(), two().clone()]
        torch.cuda.synchronize()
        a.zero_(), b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(b, want[1]), n
    del graph
    torch.cuda.synchronize()
    emu.release_workspace()
    assert emu.workspace_bytes() == 0
    emu.lib().emu_set_stream(None)
