"""Which kernels calls of the mixture-of-experts operators launch (on a stand-in for the
HIP runtime): every one that the library holds is some call's."""
import pytest

import _fake_hip as F


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


EVERY = """
import random
import _fake_hip as F
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
