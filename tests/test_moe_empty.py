"""An X without rows, which may be NULL: every row number is outside of it and stands
for a row of zeros (what the library launches, on a stand-in for the HIP runtime)."""
import pytest

import _fake_hip as F


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


@pytest.mark.parametrize("x", ["None", "F.X"])
def test_no_rows_to_read(fake, x):
    """Few rows and many, of every type; no kernel that reads a row for one outside."""
    out = F.run(fake, f"""
import _fake_hip as F
result = []
for dtype in range(3):
    for transb in "NT":
        for R in (3, 4000):
            for K in (512, 513):
                rc = L.grouped(dtype, transb, 2, R, 256, K, rows=True, XR=0, x={x})
                result.append([rc, L.kernels()])
                rc = L.wgrad(dtype, transb, 2, R, 256, K, rows=True, XR=0, x={x})
                result.append([rc, L.kernels()])
    for R in (3, 40, 4000):
        rc = L.q4(dtype, 2, R, 256, 512, rows=True, XR=0, x={x})
        result.append([rc, L.kernels()])
""")
    assert all(rc == 0 and kernels for rc, kernels in out), out
    assert not any(k.startswith(("gemm16", "wgrad16")) for _, ks in out for k in ks)


def test_refused_where_there_are_rows(fake):
    out = F.run(fake, """
result = [L.grouped(1, "N", 2, 9, 64, 64, rows=True, XR=1, x=None), L.wgrad(1, "N", 2, 9, 64, 64, rows=True, XR=1, x=None),
          L.q4(1, 2, 9, 64, 64, rows=True, XR=1, x=None), L.grouped(1, "N", 2, 9, 64, 64, XR=0)]""")
    assert out == [1, 1, 1, 1]


def test_gradient_of_the_combination_without_tokens(fake):
    """Rows of no token are cleared, whether there are tokens or not; nothing else is needed."""
    out = F.run(fake, """
from ctypes import c_int64 as i
def call(T, R, D, z=None, rows=F.X, dz=F.X):
    ld = i(max(1, D))
    rc = L.emu.emu_moe_combine_grad(1, i(T), i(D), 2, i(R), z, ld, z, ld, z, z, F.P(rows), F.P(dz), ld, z)
    return [rc, [l[2:6] for l in L.log() if l[0] == "launch"]]
result = [call(0, 10, 64), call(0, 100000, 64), call(0, 0, 64, rows=None, dz=None), call(0, 10, 0, dz=None),
          call(0, 10, 64, rows=None), call(0, 10, 64, dz=None)]""".replace("from ctypes", "import _fake_hip as F\nfrom ctypes"))
    assert out == [[0, [[10, 1, 1, 256]]], [0, [[4096, 1, 1, 256]]], [0, []], [0, []], [1, []], [1, []]]
