"""The token operators' binding to torch as another thread may find it at any
moment of a first call."""
import sys

import pytest

torch = pytest.importorskip("torch")

from paper_2512_08557_amd import tokens as T  # noqa: E402


def test_binding_is_whole_once_it_shows(monkeypatch):
    monkeypatch.setattr(T, "torch", None)
    monkeypatch.setattr(T, "_device", None)
    monkeypatch.setattr(T, "_stream", None)
    monkeypatch.setattr(T, "_KINDS", {})
    halves = []

    def look(frame, event, arg):
        if frame.f_code is T._bind.__code__:
            frame.f_trace_opcodes = True
            if T.torch is not None:
                if T._device is None or T._stream is None or len(T._KINDS) != 2:
                    halves.append((frame.f_lineno, T._device, T._stream, len(T._KINDS)))
            return look
        return None

    before = sys.gettrace()
    sys.settrace(look)
    try:
        T._bind()
    finally:
        sys.settrace(before)
    assert not halves, halves
    assert T.torch is torch and T._KINDS == {torch.float32: T.F32, torch.bfloat16: T.BF16}
