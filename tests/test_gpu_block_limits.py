"""The block operators on the GPU at the ends of what they take: arguments near the types' largest."""
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
