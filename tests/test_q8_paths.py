"""One result of an 8-bit product, whichever kernel forms it: the bits of a row of Y go by
its sums and scales alone, not by how many rows are computed with it, nor by whether the workspace
could grow.  Results are those of `Y = (float)sum * ws * xs` in FP32, rounded to the type."""
import math

import pytest
import torch

import _fake_hip as F
import _moe as M

# Rows, experts, N, K of products and the kernel that forms their results: sums up to 2^26, so that
# their conversion to FP32 rounds too
FEW, TILES, COPIED, SPLIT_FEW, SPLIT_TILES = (
    (5, 1, 300, 4096), (2000, 1, 300, 4096), (2500, 1, 300, 4095), (50, 1, 33, 40007), (130, 1, 260, 20016))
# N and K of 2000 rows: on tiles, whole and broken ones, and in splits
ENDS = [(512, 4096), (300, 4096), (256, 8128), (300, 8128)]


def test_what_forms_them(tmp_path):
    """Each of the shapes above runs what it stands for, without workspace the others."""
    got = F.run(F.build(tmp_path), f"""
from ctypes import c_int64 as i
import _fake_hip as F
p = F.P(F.X)
def gemm(R, E, N, K):
    assert L.emu.emu_q8_gemm(0, E, i(R), i(N), i(K), p, i(K), p, i(R), None, p, i(K), i(0), p, None, p, i(N)) == 0
    return [k.split("<")[0] for k in L.kernels()]
result = [gemm(*s) for s in {[FEW, TILES, COPIED, SPLIT_FEW, SPLIT_TILES]!r}]
result += [gemm(2000, 1, *s) for s in {ENDS!r}]
assert L.emu.emu_release_workspace() == 0
L.fake.fake_room(0)
result += [gemm(*s) for s in {[COPIED, SPLIT_FEW, SPLIT_TILES]!r}]
""")
    assert got == [["q8_few_kernel"], ["q8_tiles_kernel"], ["q8_copy_kernel", "q8_tiles_kernel"],
                   ["q8_few_kernel", "q8_join_kernel"], ["q8_tiles_kernel", "q8_join_kernel"],
                   ["q8_tiles_kernel"], ["q8_tiles_kernel"], ["q8_tiles_kernel", "q8_join_kernel"],
                   ["q8_tiles_kernel", "q8_join_kernel"], ["q8_few_kernel"], ["q8_few_kernel"], ["q8_few_kernel"]]


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


def _operands(R, E, N, K):
    gen = torch.Generator(device="cuda").manual_seed(K)
    ints = lambda *s: torch.randint(60, 128, s, generator=gen, device="cuda", dtype=torch.int8)  # noqa: E731
    f = lambda *s: torch.rand(s, generator=gen, device="cuda") + 0.5                             # noqa: E731
    return ints(R, K), f(R), ints(N, K), f(N)


def _same(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def _formula(X, xs, W, ws):
    """The sums in FP64, exact, then FP32 and the type as the formula says."""
    return ((X.double() @ W.double().T).float() * ws) * xs[:, None]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K", [FEW, TILES, COPIED, SPLIT_FEW, SPLIT_TILES])
def test_the_formula(emu, kind, R, E, N, K):
    X, xs, W, ws = _operands(R, E, N, K)
    dt = M.TYPES[kind]
    xs = xs * 2.0 ** -14                                    # within half's range
    assert torch.equal(emu.q8_gemm(X, xs, W, ws, dtype=dt), _formula(X, xs, W, ws).to(dt))


@pytest.mark.gpu
@pytest.mark.parametrize("R,E,N,K", [TILES, COPIED, SPLIT_FEW, SPLIT_TILES])
def test_rows_alone_and_in_a_batch(emu, R, E, N, K):
    X, xs, W, ws = _operands(R, E, N, K)
    whole = emu.q8_gemm(X, xs, W, ws, dtype=torch.float32)
    for n in (1, 5, 40):
        assert torch.equal(emu.q8_gemm(X[:n], xs[:n], W, ws, dtype=torch.float32), whole[:n])


@pytest.mark.gpu
@pytest.mark.parametrize("R,E,N,K", [COPIED, SPLIT_FEW, SPLIT_TILES])
def test_with_and_without_workspace(emu, R, E, N, K):
    """An eager call and a captured one that finds no workspace."""
    args = _operands(R, E, N, K)
    eager = emu.q8_gemm(*args, dtype=torch.float32)
    torch.cuda.synchronize()
    emu.release_workspace()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = emu.q8_gemm(*args, dtype=torch.float32)
    assert emu.workspace_bytes() == 0
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", ENDS)
def test_scales_at_the_ends_of_the_range(emu, N, K):
    """Scales whose product with a sum leaves FP32's range before the result does, subnormal
    results, scales that are not finite: the same bits in tiles (whole ones and others, plain
    scales beside extreme ones), of few rows and of splits."""
    X, xs, W, ws = _operands(2000, 1, N, K)
    xs = xs * 2.0 ** torch.linspace(-140, 30, 2000, device="cuda").round()
    xs[7], xs[9], xs[11] = math.nan, math.inf, 0.0
    ws[128] = 2.0 ** -120
    plain = emu.q8_gemm(X, xs, W, ws, dtype=torch.float32)
    assert ((plain != 0) & (plain.abs() < 2.0 ** -126)).any()
    ws[:5] = torch.tensor([2.0 ** 120, 1.7 * 2.0 ** -140, 2.0 ** -149, 0.0, 3.0 * 2.0 ** 97])
    ws[9], ws[140] = math.inf, math.nan
    whole = emu.q8_gemm(X, xs, W, ws, dtype=torch.float32)
    keep = [n for n in range(N) if n not in (0, 1, 2, 3, 4, 9, 140)]
    assert _same(whole[:, keep], plain[:, keep])
    for a, b in ((0, 1), (3, 20), (100, 150), (7, 200), (1250, 1544)):
        assert _same(emu.q8_gemm(X[a:b], xs[a:b], W, ws, dtype=torch.float32), whole[a:b])
    # a row that X does not have changes nothing for the others of its tile
    rows = torch.arange(2000, dtype=torch.int32, device="cuda")
    rows[300] = -1
    got = emu.q8_gemm(X, xs, W, ws, rows=rows, dtype=torch.float32)
    assert (got[300] == 0).all()
    assert _same(got[rows >= 0], whole[rows >= 0])
