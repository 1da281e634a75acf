"""The numbers of a stage's and an entry's dropouts: one for each place, micro-batch and training step.  No GPU."""
import types

import pytest
import torch

from paper_2311_15269_amd import block_ops, stage


class OnGpu(torch.Tensor):
    """a tensor that says it is on GPU number 0"""
    is_cuda = True

    def get_device(self):
        return 0


def numbers(monkeypatch, step, layers, microbatches):
    """of the dropouts of a training step, forward and backward"""
    drawn = []
    monkeypatch.setattr(block_ops, "dropout", lambda y, drop: drawn.append(drop))
    for mu in microbatches:
        for layer in layers:
            for which in (0, 1):
                for _ in range(2):
                    stage.Stage._drop(types.SimpleNamespace(rate=0.5, seed=7, layer=layer, step=step), None, mu, which)
        drawn += [stage.Entry._drop(types.SimpleNamespace(rate=0.5, seed=7, step=step), mu) for _ in range(2)]
    assert all(d.step is step and d.seed == 7 and d.rate == 0.5 for d in drawn)
    assert all(a.number == b.number for a, b in zip(drawn[::2], drawn[1::2]))        # (the backward pass draws what the forward pass drew)
    return [d.number + (0 if step is None else int(step)) for d in drawn[::2]]


def test_every_step_draws_anew(monkeypatch):
    step, seen = torch.zeros(1, dtype=torch.int64).as_subclass(OnGpu), []
    layers, microbatches = (0, 1, 2, 2046), (0, 1, 5, (1 << 20) - 1)
    for k in (0, 1, 2, 3, 4, 1000, (1 << 32) - 1):
        step.fill_(k)
        seen += numbers(monkeypatch, step, layers, microbatches)
    assert len(set(seen)) == len(seen) == 7 * 4 * 9 and 0 <= min(seen) and max(seen) < 1 << 64


def test_without_a_step_the_numbers_are_what_they_were(monkeypatch):
    got = numbers(monkeypatch, None, (0, 3), (0, 6))
    assert got == [mu << 32 | place for mu in (0, 6) for place in (0, 1, 6, 7, 0xFFFFFFFF)]


def test_layers_that_a_step_does_not_tell_apart_are_refused():
    with pytest.raises(ValueError):
        stage.Stage(128, 4, 2, 256, None, torch.bfloat16, rate=0.1, layer=2047, step=torch.zeros(1, dtype=torch.int64))
