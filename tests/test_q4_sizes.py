"""Sizes that the 4-bit product takes: every one whose launch fits, none that does not
(on a stand-in for the HIP runtime)."""
import pytest

import _fake_hip as F


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


def test_prompts_through_wide_matrices(fake):
    """Many rows and many columns, each within the limits of the header."""
    out = F.run(fake, """
result = [L.q4(dtype, E, R, N, 4096) for dtype in range(3)
          for E, R, N in ((1, 65536, 32768), (1, 16384, 150000), (64, 131072, 16384), (8, 1 << 20, 8192))]""")
    assert out == [0] * len(out)


def test_every_launch_fits(fake):
    """Below 2^32 threads along an axis, or refused; and refused only where X, Q and
    Y would take half of the memory of a card."""
    out = F.run(fake, """
result = []
for dtype in range(3):
    for E in (1, 7, 64, 3000, 65536):
        for R in [1 << i for i in range(0, 31, 3)] + [(1 << 31) - 1]:
            for N in [1 << i for i in range(0, 30, 3)] + [(1 << 30) - 1]:
                for K in (64, 8192):
                    rc = L.q4(dtype, E, R, N, K)
                    result.append([dtype, E, R, N, K, rc, [l[2:6] for l in L.log() if l[0] == "launch"]])
""")
    taken = 0
    for dtype, E, R, N, K, rc, launches in out:
        assert rc in (0, 1)
        taken += rc == 0
        for x, y, z, threads in launches:
            assert x * threads < 1 << 32 and y * z < 65536, (dtype, E, R, N)
        if rc == 1:
            assert R * (N + K) * (4 if dtype == 0 else 2) + E * N * K // 2 >= 1 << 37, (dtype, E, R, N, K)
    assert taken > 1500
