"""What a transformer stage promises of itself: gradients of all weights summed in 32 bits, no 8 bits where it keeps 16, and the bytes that it
holds between forward and backward."""
import pytest
import torch

pytestmark = pytest.mark.gpu
LENGTHS = [300, 1, 83]


@pytest.fixture(scope="module")
def stage():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import stage
    return stage


@pytest.mark.parametrize("small", [True, False])
def test_all_gradients_of_weights_are_sums_in_32_bits(stage, small):
    """two micro-batches: each weight's gradient is the sum of dy^T x of what its products were given, terms exact and added in 32 bits (n 2^-24 of
    their sizes at worst)"""
    from paper_2311_15269_amd import block_ops
    (s,), packings, xs, hs = stage.make(1, 2, LENGTHS, 128, 4, 2, 256, small, seed=3)
    want, size, n = {}, {}, 2 * sum(LENGTHS)
    add = s._add

    def recorded(name, dy, x):
        held = (block_ops.restore(x) if isinstance(x, block_ops.Checkpoint) else x).double().cpu()
        d = dy.double().cpu()
        want[name] = want.get(name, 0) + d.T @ held
        size[name] = size.get(name, 0) + d.abs().T @ held.abs()
        add(name, dy, x)
    s._add = recorded
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    for mu in range(2):
        r, h = s.forward(mu, packings[mu], xs[mu], hs[mu])
        s.backward(mu, *(torch.randn(r.shape, generator=gen, device="cuda").bfloat16() for _ in range(2)))
    assert sorted(want) == sorted(s.weights)
    for name, g in s.gradients.items():
        off = (g.double().cpu() - want[name]).abs() - (n + 16) * 2.0 ** -24 * size[name]
        assert g.dtype == torch.float32 and float(off.max()) <= 0.0, (name, float(off.max()))


def test_a_stage_of_16_bits_holds_nothing_in_8(stage, monkeypatch):
    from paper_2311_15269_amd import block_ops
    (s,), (packing,), (x,), (h,) = stage.make(1, 1, LENGTHS, 128, 4, 2, 256, False, seed=5)

    def refuse(*args, **more):
        raise AssertionError("8 bits")
    for name in ("checkpoint", "gated", "gated_backward", "weight_gradient"):
        monkeypatch.setattr(block_ops, name, refuse)
    r, hr = s.forward(0, packing, x, h)
    assert not any(isinstance(t, block_ops.Checkpoint) for t in s.kept[0])
    s.backward(0, r, hr)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_the_gated_part_of_a_stage_of_16_bits(stage, act):
    """the activation and its gradients from g and u as they are, rounded once each: 2^-8 of the value, and 1e-5 of the factors' sizes for 32 bits"""
    (s,), (packing,), (x,), (h,) = stage.make(1, 1, LENGTHS, 128, 4, 2, 256, False, seed=6)
    s.act = act
    gen = torch.Generator().manual_seed(7)
    g, u, da = (torch.randn(50, 256, generator=gen).bfloat16() for _ in range(3))
    x, y = g.double().requires_grad_(), u.double().requires_grad_()
    f = torch.nn.functional.silu(x) if act == "silu" else torch.nn.functional.gelu(x, approximate="tanh")
    a = f * y
    wg, wu = torch.autograd.grad(a, [x, y], da.double())
    got = (s._gated(g.cuda(), u.cuda())[0], *s._gated_backward(da.cuda(), g.cuda(), u.cuda())[:2])
    for p, q in zip(got, (a.detach(), wg, wu)):
        assert p.dtype == torch.bfloat16
        off = (p.double().cpu() - q).abs() - 2.0 ** -8 * q.abs() - 1e-5 * (1 + g.double().abs()) ** 2 * (1 + u.double().abs()) * (1 + da.double().abs())
        assert float(off.max()) <= 0.0


@pytest.mark.parametrize("small", [True, False])
def test_kept_bytes_are_what_the_stage_holds(stage, small):
    """all that stays on the GPU from a forward pass to its backward pass, its input of the residual stream among it (the stage before does not
    keep that): against what the allocator has given away, which rounds each of some twenty tensors up to 512 bytes"""
    (s,), (packing,), (x,), (h,) = stage.make(1, 1, LENGTHS, 128, 4, 2, 256, small, seed=8)
    s.backward(0, *s.forward(0, packing, x, h))                 # (what libraries keep for themselves is there now)
    torch.cuda.synchronize()
    empty = torch.cuda.memory_allocated()
    x2, h2 = x.clone(), h.clone()
    out = s.forward(1, packing, x2, h2)
    del x2, h2, out
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated() - empty
    assert held - 20 * 512 <= s.kept_bytes(1) <= held
    s.backward(1, x, h)
