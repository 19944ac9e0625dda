"""The workspace that a graph uses outlives its replacement by a larger one (a stand-in
for the HIP runtime, no GPU)."""
import pytest

import _fake_hip as F


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


CAPTURED = ["L.sgemm()", "L.grouped(1, 'N', 2, 4000, 1000, 2001)", "L.route()", "L.q4(1, 1, 16, 2048, 16384)"]


@pytest.mark.parametrize("captured", CAPTURED)
@pytest.mark.parametrize("set_before", [False, True])
@pytest.mark.parametrize("larger", ["L.sgemm(4096, 4096, 4096)", "L.grouped(1, 'N', 2, 8000, 3001, 8001)"])
def test_kept_until_the_release(fake, captured, larger, set_before):
    """Whether the stream was set before the capture began or under it."""
    begin = "L.stream(16)\nL.fake.fake_capture(16, 7)\n" if set_before else "L.fake.fake_capture(16, 7)\nL.stream(16)\n"
    held, grown, released, again, out = F.run(fake, f"""
assert {captured} == 0
held = [l for l in L.log() if l[0] == "malloc"][-1][1]
{begin}assert {captured} == 0 and L.log()
L.fake.fake_capture(16, 0)
assert L.stream(0) == 0
L.log()
assert {larger} == 0
grown = L.log()
assert {larger.replace("8000", "20000").replace("4096", "8192")} == 0
again = L.log()
assert L.emu.emu_release_workspace() == 0
result = [held, grown, L.log(), again, L.fake.fake_held()]""")
    new = [l[1] for l in grown + again if l[0] == "malloc"]
    assert len(new) == 2
    freed = [l[1] for l in grown + again if l[0] == "free"]
    assert freed == new[:1]                             # no graph uses that one
    assert sorted(l[1] for l in released if l[0] == "free") == sorted([held, new[1]]) and out == 0


def test_not_kept_without_a_capture(fake):
    log = F.run(fake, "L.stream(16); L.sgemm(); L.sgemm(512, 512, 512); result = L.log()")
    assert [l[0] for l in log if l[0] in ("malloc", "free")] == ["malloc", "free", "malloc"]


def test_status_bits_of_a_graph(fake):
    """What a graph reports after the workspace has grown is read, and cleared."""
    first, second = F.run(fake, """
import ctypes
L.sgemm(); L.stream(16); L.fake.fake_capture(16, 7); L.sgemm(); L.fake.fake_capture(16, 0)
old = [l for l in L.log() if l[0] == "malloc"][0][1]
L.sgemm(1024, 1024, 1024)
ctypes.c_uint.from_address(old).value = 8           # what the graph's split would set
flags = ctypes.c_uint()
result = []
for _ in range(2):
    assert L.emu.emu_domain_status(ctypes.byref(flags)) == 0
    result.append(flags.value)""")
    assert (first, second) == (8, 0)
