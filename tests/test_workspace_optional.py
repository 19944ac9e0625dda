"""Operators that can do without the workspace, where it cannot grow: what is held
stays, the call goes on without, nothing is tried twice; an error of the runtime is
an error of the call (a stand-in for the runtime, no GPU)."""
import pytest

import _fake_hip as F

EHIP, ENOMEM = 2, 3
# a product on copies, a gradient in pieces, 4 bits with a split reduction: the call,
# its kernels with the workspace, and without
CALLS = {
    "product": ("L.grouped(1, 'N', 2, 4000, 1000, 2001)",
                ["realign_kernel", "realign_kernel", "gemm16_kernel"], ["staged_gemm_kernel"]),
    "wgrad": ("L.wgrad(0, 'N', 4, 5000, 86, 338)", ["staged_wgrad_kernel", "join_kernel"], ["staged_wgrad_kernel"]),
    "q4": ("L.q4(1, 1, 16, 2048, 16384)", ["q4_gemm_kernel", "q4_join_kernel"], ["q4_gemm_kernel"]),
}


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


def _steps(fake, *steps):
    out = F.run(fake, "result = []\n" + "".join(
        f"rc = {step}\nresult.append([rc, L.log(), L.emu.emu_workspace_bytes()])\n" for step in steps))
    return [(rc, [l for l in log if l[0] != "launch"], [F.short(l[6]).split("<")[0] for l in log if l[0] == "launch"],
             size) for rc, log, size in out]


@pytest.mark.parametrize("call", list(CALLS))
def test_grows_where_it_can(fake, call):
    step, kernels, _ = CALLS[call]
    first, one, two = _steps(fake, "L.sgemm()", step, step)
    assert one[0] == two[0] == 0 and one[2] == two[2] == kernels
    assert one[3] > first[3] and two[1] == []
    # the held one goes when the new one is there
    assert [l[0] for l in one[1]] == ["ask", "malloc", "synchronize", "memcpy", "memcpy", "free"]


@pytest.mark.parametrize("call", list(CALLS))
def test_no_memory(fake, call):
    """Another call's workspace stays as it is, and the refused size is not asked for again."""
    step, _, kernels = CALLS[call]
    first, one, two, same = _steps(fake, "L.sgemm()", "L.fake.fake_room(L.fake.fake_held()) and 0 or " + step, step,
                                   "L.sgemm()")
    assert one[0] == two[0] == 0 and one[2] == two[2] == kernels
    assert [l[0] for l in one[1]] == ["ask"] and two[1] == [] and same[1] == []
    assert one[3] == two[3] == first[3]


@pytest.mark.parametrize("call", list(CALLS))
def test_a_size_that_was_refused_before(fake, call):
    """A size that the device could not give another call is not asked for, until a release."""
    step, kernels, without = CALLS[call]
    small, one, _, again = _steps(fake, "L.fake.fake_room(1 << 16) and 0 or L.sgemm(128, 128, 32)", step,
                                  "L.fake.fake_room(1 << 34) and 0 or L.emu.emu_release_workspace()", step)
    assert small[0] == ENOMEM and one[0] == 0 and one[2] == without and one[1] == []
    assert again[0] == 0 and again[2] == kernels


@pytest.mark.parametrize("call", list(CALLS))
def test_under_capture(fake, call):
    """No synchronisation, allocation or release may be recorded or tried there."""
    step, kernels, without = CALLS[call]
    first, one, two = _steps(fake, "L.sgemm()", "L.fake.fake_capture(16, 7) or L.stream(16) or " + step,
                             "L.fake.fake_capture(16, 0) or " + step)
    assert one[0] == 0 and one[2] == without and one[1] == [] and one[3] == first[3]
    assert two[0] == 0 and two[2] == kernels and two[3] > first[3]


def test_a_call_that_needs_it_under_capture(fake):
    first, one, two = _steps(fake, "L.sgemm()", "L.fake.fake_capture(16, 7) or L.stream(16) or L.sgemm(512, 512, 512)",
                             "L.sgemm()")
    assert one[0] == ENOMEM and one[1] == one[2] == [] and one[3] == first[3]
    assert two[0] == 0 and two[2]                       # what is held may be used


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("function", ["hipStreamSynchronize", "hipMemcpy", "hipMemset", "hipMalloc"])
def test_errors_of_the_runtime(fake, call, function):
    """Work that failed before (first told of by the synchronisation), or another error:
    the call says so and launches nothing; what was held stays."""
    step, kernels, _ = CALLS[call]
    first, one, two = _steps(fake, "L.sgemm()", f"L.fake.fake_fail(b'{function}', 719) or " + step,
                             f"L.fake.fake_fail(b'{function}', 0) or " + step)
    assert one[0] == EHIP and one[2] == [] and one[3] == first[3]
    assert two[0] == 0 and two[2] == kernels


@pytest.mark.parametrize("call", list(CALLS))
def test_limit(fake, call, monkeypatch):
    step, _, kernels = CALLS[call]
    monkeypatch.setenv("EMU_WORKSPACE_LIMIT", "4096")
    one, = _steps(fake, step)
    assert one[0] == 0 and one[2] == kernels and one[1] == [] and one[3] == 0
