"""CPU test of what becomes of the buffer that a moved cache leaves: torch must not hand
its memory out while the copy still reads it."""
import types

import pytest


class Buffer:
    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream)


@pytest.fixture
def hw(monkeypatch):
    from paper_2609_02029_amd import hwkv
    calls = []

    def move(handle, pages, ptr, n, stream):
        calls.append(stream)
        return hwkv.OK if pages >= 0 else hwkv.EINVAL

    lib = types.SimpleNamespace(hwkv_cache_move=move, hwkv_last_error=lambda: b"no")
    monkeypatch.setattr(hwkv, "_lib", lib)
    monkeypatch.setattr(hwkv, "_on_current_device", lambda *a: None)
    monkeypatch.setattr(hwkv, "_dev", lambda *a: None)
    capturing = []
    monkeypatch.setattr(hwkv.torch._C, "_cuda_isCurrentStreamCapturing", lambda: bool(capturing), raising=False)
    monkeypatch.setattr(hwkv.torch.cuda, "ExternalStream", lambda s: ("external", s))
    monkeypatch.setattr(hwkv.torch.cuda, "default_stream", lambda: "default")
    monkeypatch.setattr(hwkv.torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(hwkv, "_stream_objects", {})
    monkeypatch.setattr(hwkv, "_stream", lambda s: 77 if s is None else s if isinstance(s, int) else s.cuda_stream)
    return types.SimpleNamespace(hwkv=hwkv, calls=calls, capturing=capturing)


def test_the_left_buffer_waits_for_the_move(hw):
    cache = hw.hwkv.Cache(None, 1, 1, 1, 64, 1)
    side = types.SimpleNamespace(cuda_stream=5)
    for stream, seen, raw in ((side, ("external", 5), 5), (None, ("external", 77), 77), (9, ("external", 9), 9), (0, "default", 0)):
        left = cache.dev_buf = Buffer()
        hw.hwkv.cache_move(cache, 4, None, stream=stream)
        assert left.streams == [seen] and hw.calls[-1] == raw and cache.dev_buf is None
    left = cache.dev_buf = Buffer()
    with pytest.raises(hw.hwkv.HwkvError):
        hw.hwkv.cache_move(cache, -1, None, stream=side)
    assert cache.dev_buf is left and left.streams == []
    cache.dev_buf = None                      # the library's own buffer: freed by the call
    hw.hwkv.cache_move(cache, 4, None, stream=side)
    assert cache.left == []


def test_a_captured_move_keeps_what_replays_read(hw):
    cache = hw.hwkv.Cache(None, 1, 1, 1, 64, 1)
    left = cache.dev_buf = Buffer()
    hw.capturing.append(1)
    new = types.SimpleNamespace(numel=lambda: 8)
    hw.hwkv.cache_move(cache, 4, new, stream=3)
    assert cache.left == [left] and left.streams == [] and cache.dev_buf is new
