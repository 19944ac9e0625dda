"""Sizes that the 8-bit product takes: all within the limits of the header whose operands a card
holds, each launch below 2^32 threads (on a stand-in for the HIP runtime); the largest counts of rows
and columns on the GPU."""
import pytest
import torch

import _fake_hip as F


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


def test_every_launch_fits(fake):
    """Refused only where the rows of X that are read (one for all of Y's, at least), the matrices
    (one for all experts) and Y would take half of the memory of a card."""
    out = F.run(fake, """
import _fake_hip as F
from ctypes import c_int64 as i
p = F.P(F.X)
result = []
for dtype in (0, 1):
    for E in (1, 7, 64, 3000, 65536):
        for R in [1 << i for i in range(0, 31, 3)] + [(1 << 31) - 1]:
            for N in [1 << i for i in range(0, 30, 3)] + [(1 << 30) - 1]:
                for K in (1, 16, 77, 4096):
                    for shared in (False, True):
                        rc = L.emu.emu_q8_gemm(dtype, E, i(R), i(N), i(K), p, i(K), p, i(1 if shared else R),
                                               p if shared else None, p, i(K), i(0 if shared or E == 1 else N * K), p,
                                               p, p, i(N))
                        result.append([dtype, E, R, N, K, shared, rc,
                                       [l[2:6] for l in L.log() if l[0] == "launch"]])
result.append(L.emu.emu_workspace_bytes())
""")
    assert 0 < out.pop() <= 1 << 33                         # the header's limit of what a call asks for
    taken = 0
    for dtype, E, R, N, K, shared, rc, launches in out:
        assert rc in (0, 1)
        taken += rc == 0
        for x, y, z, threads in launches:
            assert x * threads < 1 << 32 and y * z < 65536, (dtype, E, R, N, K)
        if rc == 1:
            held = R * N * (4 if dtype == 0 else 2) + (K if shared else R * K) + (N * K if shared else E * N * K)
            assert held >= 1 << 37, (dtype, E, R, N, K, shared)
    assert taken > 5000


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    yield E
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_most_columns(emu):
    """One row, 2^30 - 1 columns of one entry each."""
    N = (1 << 30) - 1
    gen = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randint(-128, 128, (N, 1), generator=gen, device="cuda", dtype=torch.int8)
    ws = torch.rand(N, generator=gen, device="cuda")
    X, xs = torch.full((1, 1), 113, dtype=torch.int8, device="cuda"), torch.full((1,), 0.5, device="cuda")
    Y = emu.q8_gemm(X, xs, W, ws)
    for at in range(0, N, 1 << 27):
        w = W[at:at + (1 << 27), 0].float() * 113
        assert torch.equal(Y[0, at:at + (1 << 27)], (w * ws[at:at + (1 << 27)] * 0.5).bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("K", [1, 16])
def test_most_rows(emu, K):
    """2^31 - 1 rows of Y, gathered from 1000 of X and some outside, one column."""
    R, T = (1 << 31) - 1, 1000
    gen = torch.Generator(device="cuda").manual_seed(K)
    X = torch.randint(-128, 128, (T, K), generator=gen, device="cuda", dtype=torch.int8)
    W = torch.randint(-128, 128, (1, K), generator=gen, device="cuda", dtype=torch.int8)
    xs, ws = torch.rand(T, generator=gen, device="cuda"), torch.rand(1, generator=gen, device="cuda")
    rows = torch.arange(R, dtype=torch.int32, device="cuda")
    rows %= T + 7
    Y = emu.q8_gemm(X, xs, W, ws, rows=rows)
    each = ((X.double() @ W.double().T).float() * ws * xs[:, None]).bfloat16()[:, 0]
    each = torch.cat((each, each.new_zeros(7)))
    for at in range(0, R, 1 << 28):
        assert torch.equal(Y[at:at + (1 << 28), 0], each[rows[at:at + (1 << 28)]])
