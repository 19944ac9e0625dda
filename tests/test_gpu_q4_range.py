"""4-bit products at the ends of the range: entries whose integer products leave FP32's
range though the weights' do not, infinities and NaN; against 64 bits."""
import math

import pytest
import torch

import _moe as M
from test_gpu_q4 import _bar, _cuda, _matrices, _reference

pytestmark = pytest.mark.gpu
# one workgroup or several along the reduction, waves along either axis, every tile height
SHAPES = [(1, 40, 512, 32), (3, 70, 4096, 64), (7, 33, 1024, 128), (16, 100, 16384, 64), (20, 50, 96, 32),
          (40, 300, 640, 128), (64, 48, 2048, 64), (100, 1200, 256, 32)]


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("R,N,K,group", SHAPES)
def test_large_entries(emu, kind, R, N, K, group, mins):
    """Every third row near the type's largest value; results of 2^127 at most.  The bar
    is that of the other sizes (a sum formed again has less error)."""
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(R + K)
    X = torch.randn((R, K), generator=gen).clamp(-3, 3)
    X[::3] *= 1.1e38
    X[1::3] *= 2.0 ** 117
    X = X.to(dt)
    if kind == "f32":
        X[0, ::7] = torch.finfo(torch.float32).max      # (its leading component rounds to infinity)
    Q, s, m = _matrices(gen, 1, N, K, group, dt, mins)
    s, m = s * 2.0 ** -6 / K ** 0.5, None if m is None else m * 2.0 ** -6 / K ** 0.5
    Y, S = _reference(X, Q, s, m, torch.tensor([0, R]), None)
    assert float(Y.abs().max()) < 2.0 ** 127
    got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda(), mins=_cuda(m))
    M.check(got, Y, _bar(Y, S, K, group, dt))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_large_scales(emu, kind):
    """24 s is past the range, s (q - 8) x is not."""
    dt = M.TYPES[kind]
    for R in (2, 9, 33):
        gen = torch.Generator().manual_seed(R)
        X = (torch.randn((R, 256), generator=gen) / 1000).to(dt)
        Q, s, _ = _matrices(gen, 1, 60, 256, 64, dt, False)
        s = torch.full_like(s, 3e37)
        Y, S = _reference(X, Q, s, None, torch.tensor([0, R]), None)
        M.check(emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda()), Y, _bar(Y, S, 256, 64, dt))


@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,N,K,group", SHAPES)
def test_infinities_and_nan(emu, kind, R, N, K, group, mins):
    """An infinity times each weight: its sign, NaN where the weight is zero or two
    infinities cancel; the other rows are as without it."""
    dt = M.TYPES[kind]
    gen = torch.Generator().manual_seed(N + K)
    X = torch.randn((R, K), generator=gen).to(dt)
    Q, s, m = _matrices(gen, 1, N, K, group, dt, mins)
    if mins:
        m = (s.double() * -8).to(dt)                    # some weights are zero here too
    finite, S = _reference(X, Q, s, m, torch.tensor([0, R]), None)
    W = M.unpacked(Q, s, m)[0][0]
    X[0, K // 3] = math.inf
    if R > 2:
        X[2, 5], X[2, K - 1] = -math.inf, math.inf
    if R > 10:
        X[10, 0] = math.nan
    got = emu.q4_gemm(X.cuda(), Q.cuda(), s.cuda(), mins=_cuda(m)).cpu().double()
    spoiled = [r for r in (0, 2, 10) if r < R]
    want = torch.stack([(W * X[r].double()).sum(1) for r in spoiled])
    assert torch.equal(torch.isnan(got[spoiled]), torch.isnan(want))
    there = ~torch.isnan(want)
    assert torch.equal(got[spoiled][there], want[there]) and torch.isinf(want[there]).all()
    assert there.any() and (~there).any()
    got[spoiled], finite[spoiled], S[spoiled] = 0, 0, 0
    M.check(got, finite, _bar(finite, S, K, group, dt))
