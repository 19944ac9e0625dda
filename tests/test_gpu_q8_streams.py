"""Calls of two streams one after the other, without a synchronisation between: each uses the
library's one workspace (copies of operands, sums of splits, a loss's spans), with data of its own,
and gives the bits that it gives alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    yield E
    E.lib().emu_set_stream(None)


def _product(emu, gen, R, N, K):
    ints = lambda *s: torch.randint(-128, 128, s, generator=gen, device="cuda", dtype=torch.int8)  # noqa: E731
    args = (ints(R, K), torch.rand(R, generator=gen, device="cuda"), ints(N, K),
            torch.rand(N, generator=gen, device="cuda"))
    return lambda: (emu.q8_gemm(*args),)


def _balance(emu, gen, T, E):
    x = torch.randn((T, E), generator=gen, device="cuda")
    ids = torch.topk(x, 4).indices.int().contiguous()
    return lambda: tuple(emu.moe_balance(x, ids))


def test_two_streams_in_turn(emu):
    gen = torch.Generator(device="cuda").manual_seed(1)
    # a long call first, whose copies are read for longer than the next call's launch takes
    long = _product(emu, gen, 20000, 4001, 4001)
    short = [_product(emu, gen, 3000, 700, 501), _product(emu, gen, 50, 70, 30000), _balance(emu, gen, 5000, 64),
             _product(emu, gen, 2500, 900, 333), _balance(emu, gen, 3000, 128)]
    ref_long, ref = [t.clone() for t in long()], [[t.clone() for t in f()] for f in short]
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for turn in range(4):
        a, b = (one, two) if turn % 2 == 0 else (two, one)
        got = []
        for f in short:
            with torch.cuda.stream(a):
                got_long = long()
            with torch.cuda.stream(b):
                got.append(f())
            with torch.cuda.stream(a):          # and back, behind the short one
                again = f()
            got[-1] = got[-1] + again
            got.append(got_long)
        torch.cuda.synchronize()
        for i, want in enumerate(ref):
            assert all(torch.equal(u, v) for u, v in zip(got[2 * i], want + want)), (turn, i)
            assert torch.equal(got[2 * i + 1][0], ref_long[0]), (turn, i)
