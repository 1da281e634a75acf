"""Training steps of a stage and the embedding in front of it whose dropout goes by a step on the GPU: each step draws masks of its own, which its forward and backward
passes share, eagerly and in a graph that counts up."""
import pytest
import torch

from tests import entry_reference as R
from tests import test_gpu_block_entry_stage as T

pytestmark = pytest.mark.gpu
MU = 7


@pytest.fixture(scope="module")
def stage():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import stage
    return stage


def made(stage, small=True):
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    (s,), (packing,), _, _ = stage.make(1, 1, T.LENGTHS, 128, 4, 2, 256, small, seed=T.SEED, turning=T.TURNING, rate=T.RATE, step=step)
    entry, (tokens,) = stage.make_entry(1, T.LENGTHS, 128, 300, 3, seed=T.SEED, rate=T.RATE, step=step)
    return s, packing, entry, tokens, step


def gradients(s, entry):
    return dict(s.gradients, table=torch.cat(entry.gradients), pre=entry.pre_gradient, wq=s.head_gradients[0], wk=s.head_gradients[1])


def test_masks_of_steps(stage):
    s, _, entry, _, step = made(stage)
    one = torch.ones(50, 128, dtype=torch.bfloat16, device="cuda")
    seen = []
    for k in range(3):
        step.fill_(k)
        for which in (0, 1):
            y = s._drop(one, MU, which)
            assert torch.equal(y, s._drop(one, MU, which)) and torch.equal(y.cpu(), R.dropped(one.cpu(), T.RATE, T.SEED, (MU << 44 | which << 32) + k))
            seen.append(y)
        seen.append(stage.block_ops.dropout(one, entry._drop(MU)))
    assert not any(torch.equal(a, b) for i, a in enumerate(seen) for b in seen[:i])


@pytest.mark.parametrize("small", [True, False])
def test_gradients_of_every_step(stage, small, monkeypatch):
    """against torch's differentiation in 64 bits with the masks of that step; bounds as without steps"""
    s, packing, entry, tokens, step = made(stage, small)
    gen = torch.Generator().manual_seed(6)
    dr, dh = (torch.randn(sum(T.LENGTHS), 128, generator=gen).bfloat16() for _ in range(2))
    mask, seen = T.mask, []
    for k in (0, 5):
        step.fill_(k)
        x, h = entry.forward(MU, tokens)
        r, hr = s.forward(MU, packing, x, h)
        entry.backward(MU, *s.backward(MU, dr.cuda(), dh.cuda()))
        # (the plain form names a place as it does without a step: the micro-batch above 32 bits of the place)
        monkeypatch.setattr(T, "mask", lambda n, c, number: mask(n, c, (number >> 32 << 44 | (number & 0xFFF) << 32) + k))
        wr, wh, leaf, _ = T.plain(s, entry, tokens, MU)
        assert T.off(r, wr) < 0.02 and T.off(hr, wh) < 0.02
        torch.autograd.backward([wr, wh], [dr.double(), dh.double()])
        for name, g in gradients(s, entry).items():
            assert T.off(g, leaf[name].grad) < 0.05, (k, name)
        for g in list(s.gradients.values()) + list(s.head_gradients) + [v for n in s.norm_gradients for v in n.values()] + entry.gradients + [entry.pre_gradient]:
            g.zero_()
        seen.append(r)
    assert not torch.equal(*seen)


def test_a_captured_step_of_a_stage(stage):
    """a graph that counts its step up: every replay is the eager training step of that number"""
    s, packing, entry, tokens, step = made(stage)
    d = torch.randn(sum(T.LENGTHS), 128, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()

    def training_step():
        x, h = entry.forward(MU, tokens)
        r, hr = s.forward(MU, packing, x, h)
        dx, dhx = s.backward(MU, d, d)
        entry.backward(MU, dx, dhx)
        return r, hr, dx, dhx
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        training_step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = training_step()
        step += 1
    seen = []
    for k in range(4):
        step.fill_(k)
        want = training_step()
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == k + 1 and all(torch.equal(a, b) for a, b in zip(got, want)), k
        seen.append(got[0].clone())
    assert not any(torch.equal(seen[0], t) for t in seen[1:])


def test_steps_in_the_order_of_a_schedule(stage):
    """two steps in the order of a schedule and one micro-batch after the other: the same bits"""
    sizes, more = (3, 6, T.LENGTHS, 128, 4, 2, 256, True), {"turning": T.TURNING, "rate": T.RATE}
    _, _, operations = stage.plan(3, (1.0, 2.1), 3, 9, 6, max_nr=3)
    result = []
    for ops in (operations, stage.in_turn(3, 6)):
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        stages, packings, xs, _ = stage.make(*sizes, **more, step=step)
        entry, tokens = stage.make_entry(6, T.LENGTHS, 128, 1000, 3, rate=T.RATE, step=step)
        dr, out = torch.ones_like(xs[0]), []
        for _ in range(2):
            back = stage.run(stages, packings, None, None, lambda mu, r, h: (dr, h), ops, entry, tokens)
            out.append([t for pair in back for t in pair])
            step += 1
        assert not torch.equal(out[0][0], out[1][0])
        result.append(out[0] + out[1] + entry.gradients + [entry.pre_gradient] + [t for s in stages for t in (*s.gradients.values(), *s.head_gradients)])
    assert all(torch.equal(a, b) for a, b in zip(*result))


@pytest.mark.parametrize("which", [None, "weights", "norms", "heads", "shards", "entry"])
def test_the_command_compares_all_gradients(stage, which, monkeypatch, capsys):
    """one number of one of them changed on one side is a difference"""
    import sys
    monkeypatch.setattr(sys, "argv", ["stage", "--devices", "2", "--microbatches", "4", "--channels", "128", "--heads", "4", "--kv-heads", "2", "--lengths", "60,1,5", "--turning", "16",
                                      "--rate", "0.1", "--vocabulary", "300", "--steps", "2"])
    run, calls = stage.run, []

    def changed(stages, packings, xs, hs, gradient, operations, entry=None, tokens=None):
        back = run(stages, packings, xs, hs, gradient, operations, entry, tokens)
        calls.append(1)
        if which and len(calls) == 4:
            {"weights": stages[1].gradients["up"], "norms": stages[0].norm_gradients[1]["gate"], "heads": stages[1].head_gradients[0], "shards": entry.gradients[1],
             "entry": entry.pre_gradient}[which].view(-1)[3] += 1.0
        return back
    monkeypatch.setattr(stage, "run", changed)
    assert stage.main() == (1 if which else 0) and len(calls) == 4
    assert ("DIFFER" if which else "equal") in capsys.readouterr().out


def test_measuring_leaves_no_gradients(stage):
    s, packing, entry, tokens, _ = made(stage)
    x, h = entry.forward(MU, tokens)
    stage.measure(s, packing, x, h)
    assert not any(bool(g.any()) for g in s.sums()) and len(s.sums()) == len(s.gradients) + 6 + 2 and len(entry.sums()) == 4
