"""4-bit products whose workgroups take several column tiles, one after the other; every
type and tile height, with and without offsets, experts of few and of many rows."""
import pytest
import torch

import _moe as M
import _moe_shapes as S
from test_gpu_q4 import _bar, _cuda, _matrices

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K,group", S.PASSES)
def test_passes(emu, kind, R, E, N, K, group, mins):
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(R + N)
    X = torch.randn((R, K), generator=gen).to(dt).cuda()
    Q, s, m = (_cuda(t) for t in _matrices(gen, E, N, K, group, dt, mins))
    live = R - R // 10
    cuts = torch.sort(torch.randint(0, live + 1, (E - 1,), generator=gen))[0].tolist()
    at = [0, *cuts, live]
    Y = torch.full((R, N + 2), 9.0, dtype=dt, device="cuda")
    offsets = torch.tensor(at, dtype=torch.int32).cuda()
    got = emu.q4_gemm(X, Q, s, mins=m, offsets=offsets, Y=Y[:, 1:-1])
    assert (Y[:, 0] == 9).all() and (Y[:, -1] == 9).all() and (got[live:] == 0).all()
    for e in range(E):
        part = slice(at[e], at[e + 1])
        if part.start == part.stop:
            continue
        W, bound = M.unpacked(Q[e], s[e], None if m is None else m[e])
        x = X[part].double()
        exact, size = x @ W.T.contiguous(), x.abs() @ bound.T.contiguous()
        off = (got[part].double() - exact).abs()
        assert torch.isfinite(got[part]).all() and (off <= _bar(exact, size, K, group, dt)).all(), e
