"""What a call on a stream of its own allocates and fills: on that stream, or nothing would order the fill before the call's kernels.
The binding alone, with host tensors, a library that only notes its calls and streams that only have a number."""
import contextlib

import pytest
import torch

from paper_2405_14597_amd import binding


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Torch:
    """torch with fills that note the stream they are queued on."""

    def __init__(self, log):
        self.log, self.memory, self.queue = log, [], [Stream(0)]
        self.cuda = self

    def __getattr__(self, name):
        return getattr(torch, name)

    @contextlib.contextmanager
    def stream(self, s):
        self.queue.append(s)
        yield
        self.queue.pop()

    def current_stream(self):
        return self.queue[-1]

    def zeros(self, shape, dtype, device):
        self.log.append(("fill", self.queue[-1].cuda_stream))
        return self.empty(shape, dtype, device).zero_()

    def empty(self, shape, dtype, device):
        self.memory.append(self.queue[-1].cuda_stream)
        return Tensor(torch.empty(shape, dtype=dtype))


class Tensor(torch.Tensor):
    @staticmethod
    def __new__(cls, t):
        return torch.Tensor._make_subclass(cls, t)

    def record_stream(self, s):
        pass


@pytest.fixture
def log(monkeypatch):
    got = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_bytes"):
                    return 64
                got.append(("kernels", args[-1]))
                return 0
            return call

    fake = Torch(got)
    monkeypatch.setattr(binding, "_torch", lambda: fake)
    monkeypatch.setattr(binding, "load_library", lambda lib=Library(): lib)
    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: -1)
    monkeypatch.setattr(binding, "_device_of", lambda t, name: -1)
    monkeypatch.setattr(binding, "_require", lambda *a: None)
    for name, dtype in (("_half_dtype", torch.float16), ("_int32_dtype", torch.int32), ("_int64_dtype", torch.int64), ("_float_dtype", torch.float32)):
        monkeypatch.setattr(binding, name, dtype, raising=False)
    Torch.last = fake
    return got


@pytest.mark.parametrize("stream", [None, Stream(7)], ids=["current", "another"])
def test_attention_fills_a_new_output_on_its_stream(log, stream):
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    out = binding.is_attention(half(3, 128), half(3, 128), half(3, 128), torch.zeros(2, dtype=torch.int32), 64, 3, 3, stream=stream,
                               workspace=torch.zeros(64, dtype=torch.uint8))
    assert out.shape == (3, 128)
    on = 0 if stream is None else 7
    assert log == [("fill", on), ("kernels", on)]


W = torch.zeros(8, dtype=torch.uint8)
X, XQ, SA = torch.zeros((4, 128), dtype=torch.float16), torch.zeros((4, 128), dtype=torch.int8), torch.zeros(4)


def packed(floats):
    return binding.PackedWeights(W, W, 16, 128, 128, floats)


@pytest.mark.parametrize("stream", [None, Stream(7)], ids=["current", "another"])
@pytest.mark.parametrize("call", [
    lambda s: binding.is_gemm_w4a8_intscale_prepacked(XQ, SA, packed(False), None, 10, stream=s),
    lambda s: binding.is_gemm_w4a8_floatscale_prepacked(XQ, SA, packed(True), stream=s),
    lambda s: binding.is_linear_w4a8_intscale_prepacked(X, packed(False), None, 10, stream=s),
    lambda s: binding.is_linear_w4a8_floatscale_prepacked(X, packed(True), stream=s),
    lambda s: binding.is_gemm_w4a8_intscale_gate_up_silu_prepacked(XQ, SA, binding.PackedGateUp(packed(False), None, 16), 10, stream=s),
    lambda s: binding.is_gemm_w4a8_floatscale_gate_up_silu_prepacked(XQ, SA, binding.PackedGateUp(packed(True), None, 16), stream=s)],
    ids=["gemm", "gemm_float", "linear", "linear_float", "gate_up", "gate_up_float"])
def test_prepacked_calls_zero_a_new_workspace_on_their_stream(log, call, stream):
    # (the kernels count on arrival counters of zero)
    call(stream)
    on = 0 if stream is None else 7
    assert log == [("fill", on), ("kernels", on)]


half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
whole = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731


@pytest.mark.parametrize("stream", [None, Stream(7)], ids=["current", "another"])
@pytest.mark.parametrize("call,count", [
    (lambda s: binding.is_attention(half(3, 128), half(3, 128), half(3, 128), whole(2), 64, 3, 3, stream=s), 2),
    (lambda s: binding.is_qk_norm_rope(half(3, 128), half(3, 64), whole(3), torch.zeros(32), 64, v=half(3, 64), stream=s), 3),
    (lambda s: binding.is_lora_add(half(3, 64), half(2, 8, 64), half(2, 5, 8), whole(3), half(3, 5), stream=s), 2),
    (lambda s: binding.is_quantize_act_int8_token(X, stream=s), 2),
    (lambda s: binding.is_quantize_weights_int4_group(X, 128, 10, stream=s), 5),
    (lambda s: binding.is_linear_w4a8_intscale(X, W.view(1, 8).expand(16, 8), whole(16, 1), None, 128, 10, want_acc=True, stream=s), 3),
    (lambda s: binding.is_prepack_w4(torch.zeros((16, 64), dtype=torch.uint8), whole(16, 1), 128, stream=s), 2)],
    ids=["attention", "rotation", "adapters", "quantiser", "weights", "linear", "prepack"])
def test_new_tensors_are_from_the_calls_stream(log, call, count, stream):
    # (the current stream's memory may still be in use by work queued there)
    call(stream)
    assert Torch.last.memory == [0 if stream is None else 7] * count
