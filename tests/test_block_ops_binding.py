"""What block_ops refuses before the library sees it: tensors of different GPUs in one call, sizes that do not fit the structures' fields.  No GPU."""
import types

import pytest
import torch

from paper_2311_15269_amd import binding, block_ops as B

INVALID, TOOBIG = -1, -4
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


def test_lengths_that_do_not_fit_32_bits_are_refused():
    """2^32 + 5 tokens are not 5"""
    for lengths, total in (([(1 << 32) + 5], 10), ([3, -(1 << 32) + 4], 10), ([1 << 31], 10)):
        with pytest.raises(binding.TesselError):
            B.Packing(lengths, total)


def test_channels_that_do_not_fit_32_bits_are_refused():
    """2^32 + 5 channels are not 5, nor are as many outputs of a weight gradient"""
    wide = torch.zeros(1, 1, dtype=BF16).expand(1, (1 << 32) + 5)
    with pytest.raises(binding.TesselError) as error:
        B.Checkpoint(wide)
    assert error.value.code == TOOBIG
    with pytest.raises(binding.TesselError) as error:
        B.residual_norm(wide, wide, torch.ones(5))
    assert error.value.code == TOOBIG
    dy = There((1, (1 << 32) + 5), 0)
    with pytest.raises(binding.TesselError) as error:
        B.weight_gradient(dy, held((1, 64), 0))
    assert error.value.code == TOOBIG


def test_heads_that_do_not_fit_32_bits_are_refused():
    q = torch.zeros(1, 1, 8, dtype=BF16).expand(1, (1 << 32) + 2, 8)
    with pytest.raises(binding.TesselError) as error:
        B.Packing._describe(types.SimpleNamespace(_table=q, tokens=1), q, q, q, None, 0)
    assert error.value.code == TOOBIG
