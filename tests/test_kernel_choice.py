"""Which kernels calls of the mixture-of-experts operators launch (on a stand-in for the
HIP runtime): every one that the library holds is some call's."""
import pytest

import _fake_hip as F
import _moe_shapes as S


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


EVERY = """
import random
import _fake_hip as F
import _moe_shapes as S
from ctypes import c_int64 as i
p, seen = F.P(F.X), set()

def add(rc):
    assert rc == 0, L.emu.emu_last_error()
    seen.update(L.kernels())

for d in range(3):
    for T, E in ((1, 8), (100, 8), (100, 100), (100, 200), (100, 300), (100, 1000), (70000, 64)):
        add(L.route(d, T, E, 4))
        add(L.emu.emu_moe_route_grad(d, i(T), E, 4, 0, p, i(E), p, p, p, p, i(E)))
    for k in (2, 8):
        add(L.emu.emu_moe_combine(d, i(4), i(64), k, i(32), p, i(64), p, p, p, i(64)))
    add(L.emu.emu_moe_combine_grad(d, i(4), i(64), 2, i(8), p, i(64), p, i(64), p, p, p, p, i(64), p))
    add(L.emu.emu_q4_pack(d, i(4), i(64), 64, p, i(64), p, p))
    for group in (32, 64, 128):
        for R in (1, 24, 40, 400):
            for N, K in ((64, 128), (64, 16384)):
                add(L.q4(d, 1, R, N, K, group))
rng = random.Random(1)
for _ in range(60000):
    E, R = rng.choice([1, 2, 4, 8, 13, 32, 64, 200]), int(2 ** rng.uniform(0, 18))
    N, K = (int(2 ** rng.uniform(0, 13.5)) for _ in range(2))
    N, K = (n if rng.random() < 0.7 else n // 64 * 64 + 64 for n in (N, K))
    rows = rng.random() < 0.7
    call = L.grouped if rng.random() < 0.5 else L.wgrad
    add(call(rng.randrange(3), rng.choice("NT"), E, R, N, K, rows, rng.choice([max(1, R // 4), 2 * R]) if rows else None))
result = [sorted(seen), L.all_kernels()]
"""


def test_every_kernel_is_launched_by_some_call(fake):
    seen, held = F.run(fake, EVERY)
    ours = [k for k in held if k.startswith(("route_", "combine_", "few_", "gemm16", "wgrad16", "staged", "q4_",
                                             "realign", "join"))]
    assert len(ours) > 150 and [k for k in ours if k not in seen] == []


def _launches(fake, calls):
    """(kernel, workgroups) of the launches of each call, and a plan's numbers."""
    out = F.run(fake, "result = []\n" + "".join(
        f"assert {c} == 0\nresult.append(L.log(plans=True))\n" for c in calls))
    return [([(F.short(l[6]), l[2]) for l in log if l[0] == "launch"], [l[1:] for l in log if l[0] == "plan"])
            for log in out]


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
def test_large_products(fake, transb, rows):
    """Those of the GPU tests reach the tiles that they are there for."""
    for tile, shapes in ((256, S.TILES_256), (128, S.TILES_128)):
        several = 0
        for R, E, N, K in shapes:
            ((kernel, grid),), _ = _launches(fake, [f"L.grouped(1, '{transb}', {E}, {R}, {N}, {K}, {rows})"])[0]
            assert kernel.startswith(f"gemm16_kernel<bf16, {tile // 64}, "), (R, E, N, K)
            several += (R - R // 10) // tile * ((N + tile - 1) // tile) > grid
        assert several > 0


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("transb", ["N", "T"])
def test_strided_products(fake, transb, rows):
    for shapes, tile in ((S.TILES_256, 4), (S.TILES_128, 2)):
        for R, E, N, K in shapes:
            ldw = (K if transb == "T" else N) + 16
            got = _launches(fake, [f"L.grouped(1, '{transb}', {E}, {R}, {N}, {K}, {rows}, ldx={K + 24}, ldw={ldw}, "
                                   f"stride={ldw * ((N if transb == 'T' else K) + 3)})"])[0][0]
            assert len(got) == 1 and got[0][0].startswith(f"gemm16_kernel<bf16, {tile}")


@pytest.mark.parametrize("transb", ["N", "T"])
def test_large_gradients(fake, transb):
    for R, E, N, K in S.GRADIENTS_256:
        for rows in (False, True):
            ((kernel, grid),), _ = _launches(fake, [f"L.wgrad(2, '{transb}', {E}, {R}, {N}, {K}, {rows})"])[0]
            assert kernel == f"wgrad16_kernel<f16, 4, {(2 if transb == 'T' else 1) if rows else 0}>"
            assert E * -(-N // 256) * -(-K // 256) > grid
    for R, E, N, K in S.GRADIENTS_128:
        ((kernel, grid),), _ = _launches(fake, [f"L.wgrad(2, '{transb}', {E}, {R}, {N}, {K})"])[0]
        assert kernel == "wgrad16_kernel<f16, 2, 0>" and E * -(-N // 128) * -(-K // 128) > grid


def test_passes_of_columns(fake):
    seen = set()
    for dtype in range(3):
        for R, E, N, K, group in S.PASSES:
            ((kernel, _),), ((_, passes, _),) = _launches(fake, [f"L.q4({dtype}, {E}, {R}, {N}, {K}, {group})"])[0]
            assert passes > 1, (R, E, N, K)
            seen.add(kernel.split(",")[1])
    assert seen == {" 1", " 2", " 3", " 4"}             # every tile height


def test_copies_pieces_and_splits(fake):
    R, E, N, K = S.COPIED
    copied = _launches(fake, [f"L.grouped(1, 'N', {E}, {R}, {N}, {K})"])[0][0]
    assert [k.split("<")[0] for k, _ in copied] == ["realign_kernel", "realign_kernel", "gemm16_kernel"]
    R, E, N, K = S.PIECES
    assert "join_kernel<float>" in [k for k, _ in _launches(fake, [f"L.wgrad(0, 'N', {E}, {R}, {N}, {K})"])[0][0]]
    R, E, N, K, group = S.SPLIT
    assert _launches(fake, [f"L.q4(0, {E}, {R}, {N}, {K}, {group})"])[0][1][0][2] > 1


def test_few_rows_in_16_bits(fake):
    for R, E, N, K in S.FEW_T:
        for dtype in (1, 2):
            assert _launches(fake, [f"L.grouped({dtype}, 'T', {E}, {R}, {N}, {K})"])[0][0][0][0].startswith("few_kernel")
