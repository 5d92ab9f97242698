"""The clear side's binding without a GPU: streams, devices and wrong kinds of
argument, with the library and torch's stream and device contexts stood in for."""
import inspect

import pytest
import torch

from paper_2609_16915_amd import rosetta as R

CALLS = ["rms_norm_q8", "rms_norm", "rms_norm_backward", "quantize_rows", "dequantize_rows",
         "q8_matmul", "cross_entropy", "cross_entropy_backward"]


class Entered(Exception):
    pass


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_is_entered_however_it_is_passed(monkeypatch, name):
    """What a call allocates comes from the memory of the stream that it runs on."""
    stream = object()

    def enter(s):
        assert s is stream
        raise Entered

    monkeypatch.setattr(torch.cuda, "stream", enter)
    call = getattr(R, name)
    at = list(inspect.signature(call).parameters).index("stream")
    args = [torch.zeros(4, 64)] * at
    with pytest.raises(Entered):
        call(*args[:2], stream=stream)
    with pytest.raises(Entered):
        call(*args, stream)
    with pytest.raises(TypeError, match="stream"):
        call(*args, stream, stream=stream)


class OnDevice(torch.Tensor):
    """A tensor that says it lies on a ROCm device."""
    @staticmethod
    def __new__(cls, t, index):
        f = torch.Tensor._make_subclass(cls, t)
        f.index = index
        return f

    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index

    def new_empty(self, *args, **kw):
        return OnDevice(torch.empty(*args, **kw), self.index)


@pytest.fixture
def machine(monkeypatch):
    """Two devices, 0 the current one, and a library that notes where it is called."""
    class Machine:
        current, calls = 0, []

        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 64
            return lambda *a: self.calls.append((name, self.current, a[-1])) or 0

    m = Machine()
    m.calls = []

    class On:
        def __init__(self, index):
            self.index = index if isinstance(index, int) else index.index

        def __enter__(self):
            self.before, m.current = m.current, self.index

        def __exit__(self, *a):
            m.current = self.before

    class OnStream(On):
        def __init__(self, stream):
            super().__init__(stream.device_index)

    monkeypatch.setattr(R, "lib", lambda: m)
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch.cuda, "stream", OnStream)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: m.current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 1000 + i, raising=False)
    return m


def operands(index):
    """Arguments of every call, all on one device."""
    def on(*shape, dtype=torch.bfloat16):
        return OnDevice(torch.zeros(shape, dtype=dtype), index)

    f32, i8, i64 = torch.float32, torch.int8, torch.int64
    x, f = on(4, 64), lambda n: on(n, dtype=f32)
    return {
        "rms_norm_q8": (dict(x=x, weight=on(64), residual=on(4, 64), h=on(4, 64),
                             q=on(4, 64, dtype=i8)), dict(eps=1e-5, want_y=True)),
        "rms_norm": (dict(x=x, weight=on(64), residual=on(4, 64), y=on(4, 64)), dict(eps=1e-5)),
        "rms_norm_backward": (dict(gy=x, h=on(4, 64), weight=on(64), inv_rms=f(4), gh=on(4, 64),
                                   gx=on(4, 64), workspace=f(64)), {}),
        "quantize_rows": (dict(x=x, q=on(4, 64, dtype=i8), scale=f(4)), {}),
        "dequantize_rows": (dict(q=on(4, 64, dtype=i8), scale=f(4), out=x),
                            dict(dtype=torch.bfloat16)),
        "q8_matmul": (dict(a=on(4, 64, dtype=i8), a_scale=f(4), b=on(8, 64, dtype=i8), b_scale=f(8),
                           bias=f(8), out=on(4, 8), workspace=f(64)), {}),
        "cross_entropy": (dict(h=x, w=on(8, 64), targets=on(4, dtype=i64), workspace=f(64)), {}),
        "cross_entropy_backward": (dict(h=x, w=on(8, 64), targets=on(4, dtype=i64), lse=f(4),
                                        gloss=f(4), gh=on(4, 64), gw=on(8, 64), workspace=f(64)), {}),
    }


class Stream:
    def __init__(self, index):
        self.device_index, self.device, self.cuda_stream = index, torch.device("cuda", index), 2000 + index


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("index", [0, 1])
def test_a_call_runs_where_its_tensors_lie(machine, name, index):
    tensors, values = operands(index)[name]
    getattr(R, name)(**tensors, **values)
    assert machine.calls[-1][1:] == (index, 1000 + index) and machine.current == 0
    getattr(R, name)(**tensors, **values, stream=Stream(index))
    assert machine.calls[-1][1:] == (index, 2000 + index) and machine.current == 0


@pytest.mark.parametrize("name", CALLS)
def test_tensors_and_stream_of_one_device(machine, name):
    tensors, values = operands(1)[name]
    other, _ = operands(0)[name]
    for wrong in tensors:
        with pytest.raises(ValueError, match="device"):
            getattr(R, name)(**{**tensors, wrong: other[wrong]}, **values)
    with pytest.raises(ValueError, match="device"):
        getattr(R, name)(**tensors, **values, stream=Stream(0))
    assert not machine.calls


@pytest.mark.parametrize("name", CALLS)
def test_every_operand_has_to_be_a_tensor(machine, name):
    tensors, values = operands(0)[name]
    for wrong in tensors:
        for kind in ([1.0], 3, "x"):
            with pytest.raises(TypeError, match=wrong):
                getattr(R, name)(**{**tensors, wrong: kind}, **values)
    assert not machine.calls
