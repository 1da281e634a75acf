"""The block operators on the GPU at the ends of what they take: arguments near the types' largest, tensors that torch is asked to differentiate."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import block_ops
    return block_ops


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_of_the_largest_arguments(ops, act, dtype):
    """far from nought the activation is its argument or nought, up to the type's largest"""
    g = torch.tensor([1.5e38, 1.8e38, 2.5e38, 3.3e38], device="cuda")[:, None]
    g = torch.cat([g, -g]).to(dtype)
    u = torch.ones_like(g)
    a, kg, ku = ops.gated(g, u, act)
    dg, du, again = ops.gated_backward(u, kg, ku, act, with_output=True)
    kept = ops.restore(kg)
    assert torch.equal(a, g.clamp(min=0)) and torch.equal(again, kept.clamp(min=0)) and torch.equal(du, again)
    assert torch.equal(dg, (g > 0).to(dtype))


def test_tensors_that_want_gradients_are_refused(ops):
    """nothing here records torch's differentiation: a tensor that asks for it would silently get no gradient"""
    from paper_2311_15269_amd.binding import TesselError
    bf16 = torch.bfloat16
    q = torch.randn(20, 2, 64, device="cuda").to(bf16)
    x, w = torch.randn(20, 64, device="cuda").to(bf16), torch.ones(64, device="cuda")
    packing = ops.Packing([20])

    def wants(t):
        return t.detach().clone().requires_grad_()
    calls = [lambda t: packing.attention(t, q, q), lambda t: packing.attention(q, t, q), lambda t: packing.attention(q, q, t)]
    for call in calls:
        with pytest.raises(TesselError):
            call(wants(q))
        with torch.no_grad():
            call(wants(q))
        call(wants(q).detach())
    calls = [lambda t: ops.residual_norm(t, x, w), lambda t: ops.residual_norm(x, t, w), lambda t: ops.residual_norm(x, x, w, gate=t),
             lambda t: ops.gated(t, x), lambda t: ops.gated(x, t), lambda t: ops.checkpoint(t)]
    for call in calls:
        with pytest.raises(TesselError):
            call(wants(x))
        with torch.no_grad():
            call(wants(x))
    calls = [lambda t: ops.residual_norm(x, x, t), lambda t: ops.residual_norm(x, x, w, t), lambda t: ops.residual_norm(x, x, w, gate=t)]
    for call in calls:
        with pytest.raises(TesselError):
            call(wants(w))
        with torch.no_grad():
            call(wants(w))
    _, stats = ops.residual_norm(x, x, w)[1:]
    o, lse = packing.attention(q, q, q)
    k = ops.checkpoint(x)
    sums, weights = [torch.zeros(64, device="cuda") for _ in range(3)], torch.zeros(64, 64, device="cuda")
    calls = [lambda: packing.attention_backward(wants(q), q, q, q, o, lse), lambda: packing.attention_backward(q, q, wants(q), q, o, lse),
             lambda: ops.residual_norm_backward(wants(x), x, x, x, stats, w), lambda: ops.residual_norm_backward(x, x, x, x, stats, wants(w)),
             lambda: ops.residual_norm_backward(x, x, x, x, stats, w, into=[wants(t) for t in sums]), lambda: ops.gated_backward(wants(x), k, k),
             lambda: ops.weight_gradient(wants(x), k), lambda: ops.weight_gradient(x, k, into=wants(weights))]
    for call in calls:
        with pytest.raises(TesselError):
            call()
        with torch.no_grad():
            call()


def test_a_function_of_torch_may_be_made_of_them(ops):
    """in the passes of a torch.autograd.Function nothing is recorded, and its gradients are the operators'"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    q, k, v, d = (torch.randn(90, h, 64, generator=gen, device="cuda").to(torch.bfloat16) for h in (4, 2, 2, 4))
    packing = ops.Packing([70, 20])

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            o, lse = packing.attention(q, k, v)
            ctx.save_for_backward(q, k, v, o, lse)
            return o

        @staticmethod
        def backward(ctx, d_o):
            return packing.attention_backward(d_o, *ctx.saved_tensors)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(Attention.apply(*leaves), leaves, d)
    for a, b in zip(got, packing.attention_backward(d, q, k, v, *packing.attention(q, k, v))):
        assert torch.equal(a, b)
