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
