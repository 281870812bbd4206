"""The way from a public function to its module: one Python call, which checks the device and names the stream.  No GPU."""
import sys

import pytest
import torch

from paper_2502_13189_amd import binding


class Module:
    """In the place of a built module: hands its arguments back."""
    @staticmethod
    def plan(*args):
        return args


class OnGpu:
    """As much of a tensor as the way there looks at."""
    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


def test_one_python_call_on_the_way(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", int)  # (built-ins, int() is 0: no frames of their own)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", float, raising=False)
    frames = []

    def tracer(frame, event, arg):
        if event == "call" and frame.f_code.co_filename == binding.__file__:
            frames.append(frame.f_code.co_name)

    call = binding._caller(lambda: Module, "the module's")
    t = OnGpu(0)
    assert call("plan", t, None, 1, 2) == (1, 2, 0.0)  # loads it
    sys.setprofile(tracer)
    try:
        got = call("plan", t, None, 1, 2)
    finally:
        sys.setprofile(None)
    assert got == (1, 2, 0.0) and len(frames) == 1


def test_refusals():
    loads = []

    def load():
        loads.append(1)
        return Module

    call = binding._caller(load, "the module's")
    for _ in range(2):
        with pytest.raises(ValueError, match="the module's tensors live on a GPU"):
            call("plan", OnGpu(-1), None)
    assert loads == [1]  # once

    class Stream:
        cuda_stream, device_index = 7, 1

    with pytest.raises(ValueError, match="the stream is on GPU 1, the tensors on GPU 0"):
        call("plan", OnGpu(0), Stream())


def test_owners():
    x = torch.zeros(1)
    for call, owner in ((binding._cache_call, "the paged cache's"),
                        (binding._latent_call, "rotary positions' and latent attention's")):
        with pytest.raises(ValueError, match=owner + " tensors live on a GPU"):
            call("write", x, None)
