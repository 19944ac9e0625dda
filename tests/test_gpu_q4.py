"""Products with 4-bit matrices, and their packing, against 64 bits."""
import math

import pytest
import torch

import _moe as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


def _matrices(gen, E, N, K, group, dt, mins):
    Q = torch.randint(0, 256, (E, N, K // 2), generator=gen, dtype=torch.uint8)
    s = ((torch.rand((E, N, K // group), generator=gen) + 0.25) / max(1, K) ** 0.5).to(dt)
    m = (torch.randn(s.shape, generator=gen) / max(1, K) ** 0.5).to(dt) if mins else None
    return Q, s, m


def _reference(X, Q, s, m, offsets, rows):
    W, bound = M.unpacked(Q, s, m)
    Y, _ = M.grouped(X, W.transpose(1, 2), offsets, rows)
    S, _ = M.grouped(X.abs() if rows is None else X.abs(), bound.transpose(1, 2), offsets, rows)
    return Y, S


def _bar(Y, S, K, group, dt):
    """A group's sum has a rounding for each 8 of its terms and component, then
    a few more; K / group of them are added; one rounding to the type."""
    return 2.0 ** -23 * (3 * group / 8 + 4 + K / group) * S + M.rounded(Y, dt)


def _cuda(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,N,blocks", [(1, 1, 1), (1, 64, 3), (2, 100, 9), (7, 17, 2), (16, 130, 5),
                                        (17, 33, 1), (40, 48, 11), (70, 20, 4), (3, 257, 40)])
def test_dense(emu, kind, R, N, blocks, group, mins):
    dt, K = M.TYPES[kind], blocks * group
    gen = torch.Generator().manual_seed(R * N + K)
    X = torch.randn((R, K), generator=gen).to(dt)
    Q, s, m = _matrices(gen, 1, N, K, group, dt, mins)
    Y, S = _reference(X, Q, s, m, torch.tensor([0, R]), None)
    got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda(), mins=_cuda(m))
    M.check(got, Y, _bar(Y, S, K, group, dt))
    flat = emu.q4_gemm(X.cuda(), Q[0].cuda(), s[0].cuda(), mins=None if m is None else m[0].cuda())
    assert torch.equal(flat, got)


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K,group,mins,gather", [
    (1, 8, 64, 256, 64, True, False), (16, 4, 80, 320, 32, False, True), (100, 3, 50, 384, 128, True, True),
    (130, 70, 33, 96, 32, True, False), (60, 1, 40, 128, 64, False, True), (300, 2, 20, 1024, 128, False, False)])
def test_by_expert(emu, kind, R, E, N, K, group, mins, gather):
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(R + K)
    live = R - R // 8
    offsets = torch.cat((torch.sort(torch.randint(0, live + 1, (E,), generator=gen))[0], torch.tensor([live])))
    offsets[0] = 0
    X = torch.randn((R, K), generator=gen).to(dt)
    rows = None
    if gather:
        X = X[:max(1, R // 3)]
        rows = torch.randint(0, len(X), (R,), generator=gen).int()
        rows[live:] = -1
        if live > 1:
            rows[1] = len(X)
    else:
        X[live:] = math.nan
    Q, s, m = _matrices(gen, E, N, K, group, dt, mins)
    Y, S = _reference(X.nan_to_num() if not gather else X, Q, s, m, offsets, rows)
    got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda(), mins=_cuda(m), offsets=offsets.int().cuda(),
                      rows=_cuda(rows))
    M.check(got, Y, _bar(Y, S, K, group, dt))


def test_nothing_to_multiply(emu):
    X = torch.ones((4, 128), device="cuda")
    Q = torch.zeros((2, 10, 64), dtype=torch.uint8, device="cuda")
    s = torch.ones((2, 10, 2), device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert (emu.q4_gemm(X, Q, s, offsets=off) == 0).all()
    assert emu.q4_gemm(X[:0], Q, s, offsets=off).shape == (0, 10)


def test_every_integer_is_exact(emu):
    """One row of the identity picks each weight: s (q - 8) and s q + m without error."""
    for kind, dt in M.TYPES.items():
        K, group = 128, 32
        Q = torch.arange(256, dtype=torch.uint8).repeat(K // 2 // 4 + 1)[:64 * 16].reshape(1, 16, 64)
        s = torch.full((1, 16, 4), 0.25, dtype=dt)
        m = torch.full((1, 16, 4), -2.5, dtype=dt)
        X = torch.eye(K, dtype=dt)
        for mins in (None, m):
            W, _ = M.unpacked(Q, s, mins)
            got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda(), mins=_cuda(mins))
            assert torch.equal(got.cpu().double(), W[0].T.contiguous()), kind


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("shape,group", [((3, 32), 32), ((2, 5, 256), 64), ((1, 384), 128), ((4, 7, 96), 32)])
def test_packing(emu, kind, shape, group):
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(sum(shape))
    W = torch.randn(shape, generator=gen).to(dt)
    W.view(-1)[:group] = 0                                            # a group of zeros
    Q, s = emu.q4_pack(W.cuda(), group)
    w = W.float().unflatten(-1, (-1, group))
    ref_s = (w.abs().amax(-1) / 7).to(dt)
    assert torch.equal(s.cpu(), ref_s)
    sf = ref_s.float()[..., None]
    q = torch.where(sf > 0, torch.round(w / sf.clamp(min=1e-30)).clamp(-8, 7), 0.0).flatten(-2) + 8
    ref_q = (q[..., 0::2] + 16 * q[..., 1::2]).to(torch.uint8)
    assert torch.equal(Q.cpu(), ref_q)
    # the packed matrix is within half a scale of W, or the scale's own rounding
    back, _ = M.unpacked(Q.cpu(), s.cpu(), None)
    bar = s.cpu().double().repeat_interleave(group, -1) * (0.5 + 8 * 2.0 ** -8)
    assert ((back - W.double()).abs() <= bar).all()


def test_matrices_beyond_32_bit_offsets(emu):
    E, N, K, group = 5, 32768, 32768, 128
    Q = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda")
    s = torch.full((E, N, K // group), 2.0 ** -8, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(7)
    Q[-1] = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
    X = torch.randn((2, K), generator=gen, device="cuda").to(torch.bfloat16)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[-1] = 2
    got = emu.q4_gemm(X, Q, s, offsets=off)
    cols = torch.tensor([0, 1, 20000, N - 1])
    Y, S = _reference(X.cpu(), Q[-1:, cols.cuda()].cpu(), s[-1:, cols.cuda()].cpu(), None,
                      torch.tensor([0, 2]), None)
    M.check(got[:, cols.cuda()], Y, _bar(Y, S, K, group, torch.bfloat16))
    del Q
    torch.cuda.empty_cache()


def test_strided_rows(emu):
    gen = torch.Generator().manual_seed(3)
    X = torch.randn((9, 300), generator=gen)
    Q, s, _ = _matrices(gen, 1, 50, 256, 64, torch.float32, False)
    part = X[:, 7:263]
    Y, S = _reference(part, Q, s, None, torch.tensor([0, 9]), None)
    out = torch.full((9, 53), 3.0, device="cuda")
    emu.q4_gemm(X.cuda()[:, 7:263], Q.cuda(), s.cuda(), Y=out[:, 1:51])
    M.check(out[:, 1:51], Y, _bar(Y, S, 256, 64, torch.float32))
    assert (out[:, 0] == 3).all() and (out[:, 51:] == 3).all()
