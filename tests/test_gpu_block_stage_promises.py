"""What a transformer stage promises of itself: gradients of all weights summed in 32 bits."""
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
