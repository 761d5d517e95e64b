"""Tensors on another GPU than the current one are refused before anything is launched: no GPU needed."""
import pytest
import torch

import paper_2405_10951_amd as P
from paper_2405_10951_amd import binding


class On:
    """what the binding asks a tensor of a GPU for"""
    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index


@pytest.fixture
def second_is_current(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index)


def test_streams(second_is_current):
    assert binding._raw_stream(1) == binding._raw_stream(None) == binding._together(On(1), On(1), None) == 101
    for refused in (lambda: binding._raw_stream(0), lambda: binding._together(On(0), On(0))):
        with pytest.raises(ValueError, match="cuda:0.*current GPU is cuda:1"):
            refused()


def test_calls(second_is_current, monkeypatch):
    """every kind of call asks for its stream before the library is called"""
    class Library:
        def __getattr__(self, name):
            if name.endswith(("_floats", "_bytes")):
                return lambda *a: 1

            def called(*a):
                raise AssertionError(name)
            return called
    monkeypatch.setattr(binding, "load_library", Library)
    first = torch.zeros(4, 64)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    for call in (lambda: P.bsr_rmsnorm_forward(first, first[0]), lambda: P.bsr_layernorm_forward(first, first[0], first[0]), lambda: P.bsr_linear_ce_forward(first, first, torch.zeros(4, dtype=torch.int32)),
                 lambda: P.bsr_linear_ce_forward_backward(first, first, torch.zeros(4, dtype=torch.int32)), lambda: P.bsr_quantize8_rows(first), lambda: P.bsr_clip_grads([first], 1.0),
                 lambda: P.bsr_grad_norm([first])):
        with pytest.raises(ValueError, match="current GPU is cuda:1"):
            call()
