"""4-bit products at the sizes where the launch changes: reductions split over
workgroups, several column tiles to a workgroup, x copied ahead or staged, x at
odd elements, many rows with long reductions; against 64 bits."""
import pytest
import torch

import _moe as M
from test_gpu_q4 import _bar, _cuda, _matrices, _reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,N,K,group,mins", [
    (1, 64, 16384, 32, False), (1, 17, 33024, 128, True), (4, 48, 32768, 64, False), (5, 16, 16512, 32, True),
    (16, 100, 16384, 128, False), (33, 40, 16448, 64, False), (64, 30, 16384, 32, True), (65, 16, 20480, 128, False),
    (5, 300, 4224, 128, True), (16, 65, 8192, 64, False), (20, 128, 5120, 32, False), (48, 129, 4224, 128, True)])
def test_long_reductions(emu, kind, R, N, K, group, mins):
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(R * N + K)
    X = torch.randn((R, K), generator=gen).to(dt)
    Q, s, m = _matrices(gen, 1, N, K, group, dt, mins)
    Y, S = _reference(X, Q, s, m, torch.tensor([0, R]), None)
    Xc, Qc, sc, mc = X.cuda(), Q.cuda(), s.cuda(), _cuda(m)
    got = emu.q4_gemm(Xc, Qc, sc, mins=mc)
    M.check(got, Y, _bar(Y, S, K, group, dt))
    assert torch.equal(emu.q4_gemm(Xc, Qc, sc, mins=mc), got)


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K,group", [
    (3, 1, 70000, 128, 32), (5, 1, 33001, 256, 64), (100, 40, 1999, 192, 64), (40, 1, 40000, 64, 32),
    (300, 100, 1030, 128, 128)])
def test_many_columns(emu, kind, R, E, N, K, group):
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(R * N + K)
    X = torch.randn((R, K), generator=gen).to(dt)
    cuts = torch.sort(torch.randint(0, R + 1, (E - 1,), generator=gen))[0]
    offsets = torch.cat((torch.tensor([0]), cuts, torch.tensor([R])))
    Q, s, _ = _matrices(gen, E, N, K, group, dt, False)
    Y, S = _reference(X, Q, s, None, offsets, None)
    got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda(), offsets=offsets.int().cuda())
    M.check(got, Y, _bar(Y, S, K, group, dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R", [2, 6, 16, 37])
@pytest.mark.parametrize("first", [1, 2, 8])
def test_rows_at_any_element(emu, kind, R, first):
    dt, N, K, group = M.TYPES[kind], 50, 2048, 64
    gen = torch.Generator().manual_seed(R + first)
    wide = torch.full((R, K + 16), float("nan"), dtype=dt)
    wide[:, first:first + K] = torch.randn((R, K), generator=gen).to(dt)
    Q, s, m = _matrices(gen, 1, N, K, group, dt, True)
    Y, S = _reference(wide[:, first:first + K], Q, s, m, torch.tensor([0, R]), None)
    got = emu.q4_gemm(wide.cuda()[:, first:first + K], Q.cuda(), s.cuda(), mins=m.cuda())
    M.check(got, Y, _bar(Y, S, K, group, dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
def test_an_infinite_entry_stays_in_its_row(emu, kind):
    dt = M.TYPES[kind]
    for R in (3, 12):
        gen = torch.Generator().manual_seed(R)
        X = torch.randn((R, 512), generator=gen).to(dt)
        Q, s, _ = _matrices(gen, 1, 40, 512, 32, dt, False)
        X[1, 77] = float("inf")
        got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda()).cpu()
        assert (~torch.isfinite(got[1].float())).all()
        X[1] = 0
        Y, S = _reference(X, Q, s, None, torch.tensor([0, R]), None)
        got[1] = 0
        M.check(got, Y, _bar(Y, S, 512, 32, dt))
