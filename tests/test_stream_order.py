"""The order of calls on different streams, all of which use the one workspace: what
the library asks of the HIP runtime at each switch (a stand-in, no GPU)."""
import pytest

import _fake_hip as F

S0, C, D, S2 = 16, 32, 48, 64       # streams
EHIP = 2


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return F.build(tmp_path_factory.mktemp("fake_hip"))


def _steps(fake, *steps):
    """The events and launches of the steps: ("on", stream) sets the stream and
    makes a call, ("call",) makes one; each has a list of [what, stream, ...]."""
    script = "S0, C, D, S2 = 16, 32, 48, 64\nL.sgemm(); L.log(); result = []\n" + "".join(
        f"rc = {step}\nresult.append([rc, [l[:3] for l in L.log()]])\n" for step in steps)
    return F.run(fake, script)


def _edges(entry):
    """(waiting stream, stream waited for) of the events of a step."""
    rc, lines = entry
    recorded = {l[1]: l[2] for l in lines if l[0] == "record"}
    return [(l[1], recorded[l[2]]) for l in lines if l[0] == "wait"]


def test_a_switch_outside_of_a_capture(fake):
    out = _steps(fake, "L.stream(S0)", "L.sgemm()", "L.stream(S0)", "L.stream(S2)", "L.sgemm()")
    assert [_edges(o) for o in out] == [[(S0, 0)], [], [], [(S2, S0)], []]
    assert all(rc == 0 for rc, _ in out)


def test_two_streams_of_one_capture_follow_one_another(fake):
    """Begun on the current stream, then forked: calls on either side share the
    workspace, so the graph needs an edge between them, and one back."""
    out = _steps(fake, "L.stream(C)", "L.sgemm()", "L.fake.fake_capture(C, 7) or L.fake.fake_capture(D, 7) or L.sgemm()",
                 "L.stream(D)", "L.sgemm()", "L.stream(C)", "L.sgemm()")
    assert [_edges(o) for o in out] == [[(C, 0)], [], [], [(D, C)], [], [(C, D)], []]


def test_calls_outside_between_those_of_a_capture(fake):
    """The edge is between the capture's streams, whatever ran outside meanwhile, and
    no event crosses the capture's border."""
    out = _steps(fake, "L.stream(S0)", "L.sgemm()", "L.fake.fake_capture(C, 7) or L.fake.fake_capture(D, 7) or L.stream(C)",
                 "L.sgemm()", "L.stream(S0)", "L.sgemm()", "L.stream(S2)", "L.stream(D)", "L.sgemm()", "L.stream(S2)")
    assert [_edges(o) for o in out] == [[(S0, 0)], [], [], [], [], [], [(S2, S0)], [(D, C)], [], []]


@pytest.mark.parametrize("end", ["after", "before"])
def test_calls_after_a_capture_follow_those_before_it(fake, end):
    """A call on S0, a capture on C, a call on S2: it must wait for S0."""
    ended = "L.fake.fake_capture(C, 0) or "
    out = _steps(fake, "L.stream(S0)", "L.sgemm()", "L.fake.fake_capture(C, 7) or L.stream(C)", "L.sgemm()",
                 (ended if end == "before" else "") + "L.stream(S2)", "L.sgemm()")
    assert [_edges(o) for o in out] == [[(S0, 0)], [], [], [], [(S2, S0)], []]


@pytest.mark.parametrize("again", [False, True])
def test_a_captured_stream_used_outside_afterwards(fake, again):
    """The stream that was captured, then used outside: after the last call outside,
    whether it is set again or not, and the next stream after it."""
    out = _steps(fake, "L.stream(S0)", "L.sgemm()", "L.fake.fake_capture(C, 7) or L.stream(C)", "L.sgemm()",
                 "L.fake.fake_capture(C, 0) or " + ("L.stream(C)" if again else "0"), "L.sgemm()", "L.stream(S2)")
    edges = [_edges(o) for o in out]
    assert edges[4] + edges[5] == [(C, S0)] and edges[6] == [(S2, C)]
    # before the call's first launch
    if not again:
        assert [l[0] for l in out[5][1]][:2] == ["record", "wait"]


def test_another_capture(fake):
    """Streams of two captures are not joined to one."""
    out = _steps(fake, "L.fake.fake_capture(C, 7) or L.stream(C)", "L.sgemm()",
                 "L.fake.fake_capture(C, 0) or L.fake.fake_capture(D, 8) or L.stream(D)", "L.sgemm()")
    assert all(_edges(o) == [] for o in out)


def test_a_switch_that_fails_leaves_the_stream(fake):
    """Work outside cannot wait for a stream whose earlier work is behind a capture;
    nor where an event call fails.  The call says so and the stream stays."""
    out = _steps(fake, "L.stream(C)", "L.sgemm()", "L.fake.fake_capture(C, 7) or L.stream(S2)",
                 "L.fake.fake_capture(C, 0) or L.sgemm()")
    assert [rc for rc, _ in out] == [0, 0, EHIP, 0] and all(_edges(o) == [] for o in out[2:])
    assert all(l[1] == C for l in out[3][1] if l[0] == "launch")
    for function in ("hipEventRecord", "hipStreamWaitEvent", "hipEventCreateWithFlags", "hipStreamGetCaptureInfo"):
        out = _steps(fake, f"L.fake.fake_fail(b'{function}', 1) or L.stream(S2)",
                     f"L.fake.fake_fail(b'{function}', 0) or L.sgemm()", "L.stream(S2)", "L.sgemm()")
        assert [rc for rc, _ in out] == [EHIP, 0, 0, 0], function
        assert {l[1] for l in out[1][1] if l[0] == "launch"} == {0}, function
        assert {l[1] for l in out[3][1] if l[0] == "launch"} == {S2}, function
