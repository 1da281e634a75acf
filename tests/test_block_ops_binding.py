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


def test_positions_stay_until_the_streams_that_read_them_are_done(monkeypatch):
    """made on one stream and read on another, they are recorded there: else the first one's next tensor may get their memory while the other still reads them"""
    now, recorded = ["first"], []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: recorded.append((t.data_ptr(), stream)))
    p = object.__new__(B.Packing)
    p.lengths, p.tokens, p._table, p._positions, p._h = [2, 0, 3], 6, torch.empty(0), None, None
    at = p.positions
    assert at.tolist() == [0, 1, 0, 1, 2, 0] and p.positions is at and not recorded
    now[0] = "second"
    assert p.positions is at and recorded == [(at.data_ptr(), "second")]
    now[0] = "first"
    assert p.positions is at and len(recorded) == 1


class OnGpu(torch.Tensor):
    """a tensor that says it is on GPU number 0"""
    is_cuda = True

    def get_device(self):
        return 0


@pytest.mark.parametrize("which", range(7))
def test_rotations_refuse_whatever_requires_a_gradient(which):
    """while torch records: queries, keys, frequencies and weights alike, and what a backward call takes"""
    q, k = (torch.zeros(5, h, 8, dtype=BF16).as_subclass(OnGpu) for h in (2, 1))
    all_of = [q, k, torch.ones(4, dtype=torch.float64).as_subclass(OnGpu), *(torch.ones(8).as_subclass(OnGpu) for _ in range(2)), q.clone(), k.clone()]
    at = torch.zeros(5, dtype=torch.int64).as_subclass(OnGpu)

    def call():
        q, k, f, wq, wk, dq, dk = all_of
        B._same(q, q.shape, dq)
        B._same(q, k.shape, dk)
        return B._describe_rotation(q, k, at, f, wq, wk, 1e-6, False)
    call()
    all_of[which].requires_grad_()
    with pytest.raises(binding.TesselError) as error:
        call()
    assert error.value.code == INVALID and "gradient" in str(error.value)
    with torch.no_grad():
        call()
