"""What the binding looks up once and keeps: whole at every moment for the threads that find it, and right without torch's shortcuts."""
import sys

import pytest
import torch

from paper_2405_14597_amd import binding

KEPT = {"_device_of": ("_half_dtype", "_int32_dtype", "_int64_dtype", "_float_dtype"), "_stream_handle": ("_current_raw_stream", "_current_device")}


class Cuda:
    """The parts of torch that the binding asks for devices and streams; the current device is 3."""
    cuda_stream = 77

    def __init__(self, shortcuts):
        self.cuda = self
        self._C = type("C", (), {"_cuda_getDevice": lambda s: 3, "_cuda_getCurrentRawStream": lambda s, d: 77} if shortcuts else {})()

    def __getattr__(self, name):
        return getattr(torch, name)

    def current_stream(self):
        return self

    def current_device(self):
        return 3


class OnDevice:
    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


@pytest.fixture(params=[True, False], ids=["shortcuts", "without"])
def fresh(request, monkeypatch):
    fake = Cuda(request.param)
    monkeypatch.setattr(binding, "_torch", lambda: fake)
    for name in sum(KEPT.values(), ()):
        monkeypatch.setattr(binding, name, None)


@pytest.mark.parametrize("fn", list(KEPT))
def test_no_moment_with_a_part_of_it(fresh, fn):
    tested, rest = KEPT[fn][0], KEPT[fn][1:]
    seen = []

    def trace(frame, event, arg):
        if frame.f_code.co_name != fn:
            return None
        frame.f_trace_opcodes = True
        seen.append(getattr(binding, tested) is None or all(getattr(binding, n) is not None for n in rest))
        return trace

    sys.settrace(trace)
    try:
        binding._device_of(OnDevice(3), "q") if fn == "_device_of" else binding._stream_handle(None)
    finally:
        sys.settrace(None)
    assert len(seen) > 20 and all(seen)
    assert all(getattr(binding, n) is not None for n in KEPT[fn])


def test_tensors_on_the_current_device_whichever_it_is(fresh):
    assert binding._stream_handle(None) == 77 and binding._stream_handle(None) == 77
    assert binding._device_of(OnDevice(3), "q") == 3
    with pytest.raises(ValueError, match="current cuda device"):
        binding._device_of(OnDevice(0), "q")
