"""What block_ops refuses before the library sees it: tensors of different GPUs in one call.  No GPU."""
import types

import pytest
import torch

from paper_2311_15269_amd import binding, block_ops as B

INVALID = -1
BF16 = torch.bfloat16


class There:
    """a tensor on GPU number `at` as far as the checks look"""
    is_cuda, dtype, requires_grad = True, BF16, False

    def __init__(self, shape, at):
        self.shape, self.at, self.device = torch.Size(shape), at, "cuda:%d" % at

    def get_device(self):
        return self.at

    def stride(self):
        return (self.shape[1], 1)

    def dim(self):
        return 2

    def data_ptr(self):
        return 1 << 20


def held(shape, at):
    c = B.Checkpoint(torch.zeros(shape, dtype=BF16))
    c._at, c.device = at, "cuda:%d" % at
    return c


def test_checkpoints_of_two_gpus_are_refused(monkeypatch):
    """a gated activation's two checkpoints: the second one's GPU too is that of the gradient"""
    def refuse(*args):
        raise AssertionError("the library was called")
    monkeypatch.setattr(B, "_library", lambda: types.SimpleNamespace(tessel_gated_backward=refuse))
    monkeypatch.setattr(B, "_stream", lambda t: 0)
    monkeypatch.setattr(B, "_like", lambda t: There(t.shape, t.at))
    da = There((4, 64), 0)
    for kg, ku in ((held((4, 64), 1), held((4, 64), 1)), (held((4, 64), 0), held((4, 64), 1))):
        with pytest.raises(binding.TesselError) as error:
            B.gated_backward(da, kg, ku)
        assert error.value.code == INVALID
    with pytest.raises(AssertionError):
        B.gated_backward(da, held((4, 64), 0), held((4, 64), 0))
