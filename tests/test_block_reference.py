"""The 64-bit references of the block operators against differences and hand-worked values.  No GPU."""
import math

import torch

from tests import block_reference as R


def _difference(f, x, step=1e-6):
    """the gradient of f at x by central differences"""
    g = torch.zeros_like(x)
    for i in range(x.numel()):
        up, down = x.clone(), x.clone()
        up.view(-1)[i] += step
        down.view(-1)[i] -= step
        g.view(-1)[i] = (f(up) - f(down)) / (2 * step)
    return g


def test_attention_gradients_are_those_of_differences():
    gen = torch.Generator().manual_seed(3)
    lengths = [1, 0, 5, 3]
    n = sum(lengths) + 2
    q, k, v, d = (torch.randn(n, h, 4, generator=gen, dtype=torch.float64) for h in (4, 2, 2, 4))
    R.U[torch.float64], R.TINY[torch.float64] = 2.0 ** -52, 2.0 ** -1000
    out, _ = R.attention(q, k, v, lengths, 0.7, d)

    def loss(q, k, v):
        return float((R.attention(q, k, v, lengths, 0.7)[0]["o"] * d).sum())
    assert torch.allclose(out["dq"], _difference(lambda t: loss(t, k, v), q), rtol=1e-6, atol=1e-8)
    assert torch.allclose(out["dk"], _difference(lambda t: loss(q, t, v), k), rtol=1e-6, atol=1e-8)
    assert torch.allclose(out["dv"], _difference(lambda t: loss(q, k, t), v), rtol=1e-6, atol=1e-8)
    assert torch.equal(out["o"][-2:], torch.zeros(2, 4, 4, dtype=torch.float64)) and bool((out["lse"][:, -2:] == -math.inf).all())
    assert torch.equal(out["o"][0], v[0].repeat_interleave(2, 0))          # one key: its value


def test_norm_gradients_are_those_of_differences():
    gen = torch.Generator().manual_seed(4)
    x, y, gate, dr, dh = (torch.randn(3, 5, generator=gen, dtype=torch.float64) for _ in range(5))
    pre, post = (1 + 0.1 * torch.randn(5, generator=gen, dtype=torch.float64) for _ in range(2))
    out = R.norm(x, y, pre, post, gate, 0.5, 1e-3, dr, dh)

    def loss(**change):
        v = dict(x=x, y=y, pre=pre, post=post, gate=gate)
        v.update(change)
        o = R.norm(v["x"], v["y"], v["pre"], v["post"], v["gate"], 0.5, 1e-3)
        return float((o["r"] * dr + o["h"] * dh).sum())
    for name, value in (("x", x), ("y", y), ("pre", pre), ("post", post), ("gate", gate)):
        assert torch.allclose(out["d" + name], _difference(lambda t: loss(**{name: t}), value), rtol=1e-6, atol=1e-7), name


def test_checkpoints_by_hand():
    x = torch.zeros(5, 70, dtype=torch.bfloat16)
    x[0, 0], x[0, 1], x[0, 2] = 127.0, 0.5, 1.5                 # 2^0; ties go to the even number
    x[1, 0], x[1, 1] = 127.5, 3.0                               # does not fit 2^0: 2^1; 63.75 and 1.5
    x[2, 69] = -1.0                                             # a group of six channels: 64 x 2^-6
    x[3, 3] = math.inf
    x[4, 5] = torch.finfo(torch.bfloat16).max                   # 63.75 x 2^122 would round to 2^128
    whole, exponent = R.held(x)
    assert exponent.tolist() == [[0, -126], [1, -126], [-126, -6], [-1000, -126], [122, -126]]
    assert whole[0, :3].tolist() == [127, 0, 2] and whole[1, :2].tolist() == [64, 2] and whole[2, 69] == -64 and whole[4, 5] == 63
    y = R.values(whole, exponent)
    assert y[2, 69] == -1 and bool(y[3, :64].isnan().all()) and bool((y[3, 64:] == 0).all())
    h = torch.tensor([[65504.0] + [2.0 ** -24] * 3])
    whole, exponent = R.held(h.half())
    assert exponent.tolist() == [[10]] and whole.tolist() == [[63, 0, 0, 0]]
    whole, exponent = R.held(h[:, 1:].half())
    assert exponent.tolist() == [[-24]] and whole.tolist() == [[1, 1, 1]]


def test_activations():
    z = torch.tensor([0.0, 1.0, -30.0, 30.0], dtype=torch.float64)
    assert torch.allclose(R.act("silu", z), torch.nn.functional.silu(z))
    assert torch.allclose(R.act("gelu", z), torch.nn.functional.gelu(z, approximate="tanh"))
