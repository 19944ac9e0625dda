"""The binding where the library cannot switch to the current stream: the call raises
and launches nothing (on the previous stream)."""
import types

import pytest
import torch

import paper_2609_04663_amd as emu


@pytest.fixture
def calls(monkeypatch):
    """The library's entry points called, with a switch of streams that fails."""
    made = []
    fake = types.SimpleNamespace(
        emu_set_stream=lambda s: made.append(("stream", s)) or emu.EMU_EHIP,
        emu_last_error=lambda: b"stream switch: the previous stream is under capture")
    monkeypatch.setattr(emu, "lib", lambda: fake)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda at: 77, raising=False)
    return made


def test_operators(calls):
    with pytest.raises(emu.EmuError, match="under capture"):
        emu._launch(lambda *a: calls.append(a) or emu.EMU_OK, torch.device("cuda", 0), 1, 2)
    assert calls == [("stream", 77)]


def test_products(calls):
    with pytest.raises(emu.EmuError, match="under capture"):
        emu._bind_stream(torch.device("cuda", 0))
    assert calls == [("stream", 77)]
