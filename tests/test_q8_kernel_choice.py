"""Which kernels calls of the 8-bit operators and of the balance loss launch (on a stand-in
for the HIP runtime), and what they do without workspace."""
import pytest

import _fake_hip as F
import _q8_shapes as S

CALLS = """
import random
import _fake_hip as F
import _q8_shapes as S
from ctypes import c_int64 as i
p, seen = F.P(F.X), set()

def balance(d, T, E, S=1):
    assert L.emu.emu_moe_balance(d, i(T), E, 1, S, p, i(E), p, p if S > 1 else None, p, p, p, p) == 0
    assert L.emu.emu_moe_balance_grad(d, i(T), E, S, p, i(E), p, p, p if S > 1 else None, p, p, p, i(E)) == 0

def rows(d, R, K):
    assert L.emu.emu_q8_pack(d, i(R), i(K), p, i(K), p, i(K), p) == 0
    assert L.emu.emu_q8_unpack(d, i(R), i(K), p, i(K), p, p, i(K)) == 0

def gemm(d, R, E, N, K, gather=False, XR=None, x=F.X, ldx=None, w=F.X):
    rc = L.emu.emu_q8_gemm(d, E, i(R), i(N), i(K), F.P(x), i(ldx or K), p, i(R if XR is None else XR),
                           p if gather else None, F.P(w), i(K), i(N * K if E > 1 else 0), p, p if E > 1 else None, p,
                           i(N))
    assert rc == 0, L.emu.emu_last_error()
    return L.kernels()
"""


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


def test_every_kernel_is_launched_by_some_call(fake):
    seen, held = F.run(fake, CALLS + """
for d in range(3):
    for E in (8, 60, 100, 200, 400, 1000):
        for T, S_ in ((100, 3), (5000, 1)):
            balance(d, T, E, S_)
    for K in (100, 200, 500, 1000, 2000, 4000, 8000, 16000, 20000):
        rows(d, 10, K)
seen.update(L.kernels())
rng = random.Random(1)
for _ in range(20000):
    E, R = rng.choice([1, 1, 4, 13, 64]), int(2 ** rng.uniform(0, 17))
    N, K = (int(2 ** rng.uniform(0, 13.5)) for _ in range(2))
    K = K if rng.random() < 0.3 else K // 16 * 16 + 16
    seen.update(gemm(rng.randrange(3), R, E, N, K, rng.random() < 0.5, rng.choice([None, 2 * R])))
for _ in range(3000):
    R, N, K = (int(2 ** rng.uniform(a, b)) for a, b in ((0, 11), (0, 12), (11, 16)))
    K = K if rng.random() < 0.3 else K // 16 * 16
    seen.update(gemm(rng.randrange(3), R, 1, N, K, rng.random() < 0.5))
for _ in range(3000):                               # a few rows of large matrices
    R, N, K = (int(2 ** rng.uniform(a, b)) for a, b in ((0, 7), (11, 15), (7, 13)))
    seen.update(gemm(rng.randrange(3), R, 1, N, K if rng.random() < 0.5 else K // 4 * 4, rng.random() < 0.5))
result = [sorted(seen), L.all_kernels()]
""")
    ours = [k for k in held if k.startswith(("balance_", "q8_"))]
    assert len(ours) > 90 and [k for k in ours if k not in seen] == []


def test_shapes_of_the_gpu_tests(fake):
    """Each group reaches its kernels; together all of them."""
    few, tiles, odd, large, splits = F.run(fake, CALLS + """
result = [[[k for gather in (False, True) for k in gemm(1, *s, gather)] for s in g]
          for g in (S.FEW, S.SHAPES, S.ODD, S.LARGE, S.SPLIT)]
""")
    reached = {k for ks in few for k in ks if k.startswith("q8_few_kernel<bf16")}
    assert len(reached) == 15, reached
    reached = {k for ks in few + tiles + odd + large for k in ks if k.startswith("q8_tiles_kernel<bf16")}
    assert len(reached) == 6, reached
    assert sum("q8_copy_kernel" in ks for ks in odd) >= 2
    assert {k for ks in splits for k in ks} >= {f"q8_few_kernel<int, {m}, 1, {odd}>" for m in (1, 2, 4)
                                                for odd in ("false", "true")} | {
        "q8_tiles_kernel<int, 2, 4, false>", "q8_tiles_kernel<int, 2, 4, true>", "q8_join_kernel<bf16>"}
    assert all(any(k.startswith("q8_tiles_kernel") for k in ks) for ks in large)
    assert "q8_tiles_kernel<bf16, 2, 4, true>" in large[3]              # four stages, two tiles to a workgroup


def test_without_workspace(fake):
    """Unaligned operands of many rows are copied, and read as they are where the workspace
    cannot grow; aligned ones need none."""
    got = F.run(fake, CALLS + """
result = [gemm(1, 4000, 1, 1000, 1001), gemm(1, 4000, 1, 1000, 1024, x=F.X + 1), L.emu.emu_workspace_bytes() > 0]
assert L.emu.emu_release_workspace() == 0
L.fake.fake_room(0)
result += [gemm(1, 4000, 1, 1000, 1001), gemm(1, 4000, 1, 1000, 1024), L.emu.emu_workspace_bytes()]
result.append([gemm(1, *s) for s in S.SPLIT])
""")
    for kernels in got[:2]:
        assert kernels[0] == "q8_copy_kernel" and kernels[1].startswith("q8_tiles_kernel") and len(kernels) == 2
    assert got[2] and got[5] == 0
    assert got[3] == ["q8_few_kernel<bf16, 4, 2, true>"]
    assert len(got[4]) == 1 and got[4][0].startswith("q8_tiles_kernel")
    assert all(len(kernels) == 1 for kernels in got[6])


def test_copies_take_the_fewer_rows(fake):
    """Rows of X through their numbers: of a large X only the rows that are read are copied,
    by the workspace's size; X beyond what 32-bit offsets span is copied too."""
    small, whole, span = F.run(fake, CALLS + """
result = []
gemm(1, 2000, 1, 3000, 1000 * 2 + 1, True, 1000000)
result.append(L.emu.emu_workspace_bytes())
assert L.emu.emu_release_workspace() == 0
gemm(1, 2000, 1, 3000, 1000 * 2 + 1, True, 1500)
result.append(L.emu.emu_workspace_bytes())
result.append(gemm(1, 4000, 1, 4096, 4096, True, 1 << 21))
""")
    ld = 2016
    assert (2000 + 3000) * ld <= small < (2000 + 3000) * ld * 2
    assert (1500 + 3000) * ld <= whole < (2000 + 3000) * ld * 2
    assert span[0] == "q8_copy_kernel" and span[1].startswith("q8_tiles_kernel")
