"""Gradients of attention in half precision on the GPU where the sizes of values, gradients and probabilities differ widely: the type
holds 2^-24 to 2^16, the gradients of the scores may be anywhere.  Against the definition in 64 bits, by norms: each of the roundings on the way
(probabilities, gradients of the scores, o inside delta, results) is 2^-11 of what is rounded at most, six of them together."""
import math

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
F16 = torch.float16
SIX = 6 * 2.0 ** -11


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import block_ops
    return block_ops


def normal(gen, n, heads, dim):
    return torch.randn(n, heads, dim, generator=gen)


def gradients(ops, q, k, v, d, lengths, scale=None):
    packing = ops.Packing(lengths, q.shape[0])
    gq, gk, gv, gd = (t.cuda() for t in (q, k, v, d))
    o, lse = packing.attention(gq, gk, gv, scale)
    return dict(zip(("dq", "dk", "dv"), (t.double().cpu() for t in packing.attention_backward(gd, gq, gk, gv, o, lse, scale))))


def near(got, want, names=("dq", "dk", "dv"), share=SIX):
    for name in names:
        assert bool(got[name].isfinite().all()), name
        off, size = float((got[name] - want[name]).norm()), float(want[name].norm())
        assert off <= share * size, (name, off / size)


@pytest.mark.parametrize("lengths, heads, kv_heads, dim", [([700], 2, 1, 64), ([300, 1, 90], 2, 2, 128), ([2000], 1, 1, 64)])
@pytest.mark.parametrize("power", [-11, -6, 6, 10, 13])
def test_values_and_gradients_of_opposite_sizes(ops, lengths, heads, kv_heads, dim, power):
    """values 2^-power as large, gradients 2^power: dq and dk are the same, dv is as much larger"""
    gen, n = torch.Generator().manual_seed(21), sum(lengths)
    q, k = normal(gen, n, heads, dim).to(F16), normal(gen, n, kv_heads, dim).to(F16)
    v = ((normal(gen, n, kv_heads, dim) * 2 ** 11).round() * 2.0 ** (-11 - power)).to(F16)
    d = ((normal(gen, n, heads, dim) * 2 ** 11).round() * 2.0 ** (power - 11)).to(F16)
    want, _ = R.attention(q, k, v, lengths, dim ** -0.5, d)
    near(gradients(ops, q, k, v, d, lengths), want, ("dq", "dk", "dv") if power <= 10 else ("dq", "dk"))


@pytest.mark.parametrize("n", [2, 40, 300])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", [1000.0, 8000.0, 30000.0])
def test_large_values_along_and_against_the_gradients(ops, n, dim, size):
    """v = +-size in all channels and gradients of one sign: the gradient of a score is some dim size |do|, far inside the type's range"""
    gen = torch.Generator().manual_seed(22)
    sign = torch.randn(n, 1, 1, generator=gen).sign()
    sign[0], sign[1] = 1.0, -1.0
    q = (0.01 * normal(gen, n, 2, dim)).to(F16)
    k = (0.01 * normal(gen, n, 1, dim)).to(F16)
    v = (size * sign * (1 + 0.01 * normal(gen, n, 1, dim))).to(F16)
    d = (0.01 * (1 + 0.2 * normal(gen, n, 2, dim))).to(F16)
    d[:, 1] *= -1
    want, _ = R.attention(q, k, v, [n], dim ** -0.5, d)
    near(gradients(ops, q, k, v, d, [n]), want)


def test_two_tokens_by_hand(ops):
    """v = +-1000, do = 0.01, k = +-0.01 in 128 channels, q = 0: p = 1/2, do . v = +-1280, and so gradients of the scores of +-640"""
    one = torch.ones(1, 1, 128)
    q, d = torch.zeros(2, 1, 128, dtype=F16), (0.01 * torch.cat([one, one])).to(F16)
    k, v = torch.cat([0.01 * one, -0.01 * one]).to(F16), torch.cat([1000 * one, -1000 * one]).to(F16)
    got = gradients(ops, q, k, v, d, [2])
    c, e = float(k[0, 0, 0]), float(d[0, 0, 0])
    dq = 128 ** -0.5 * 2 * (64 * 1000 * e) * c
    assert float((got["dq"][1] - dq).abs().max()) <= 2.0 ** -10 * dq and bool((got["dq"][0].abs() <= 2.0 ** -10 * dq).all())
    assert bool((got["dk"] == 0).all())


@pytest.mark.parametrize("dim", [64, 128])
def test_scores_gradients_that_grow_and_shrink_along_a_sequence(ops, dim):
    """values from 2^-10 to 2^10 in one sequence, growing or shrinking: every query's and every key's sums keep their digits"""
    gen, n = torch.Generator().manual_seed(23), 500
    for step in (20.0 / n, -20.0 / n):
        size = torch.exp2(step * (torch.arange(n, dtype=torch.float32) - n / 2))[:, None, None]
        q, k, d = (normal(gen, n, h, dim).to(F16) for h in (2, 1, 2))
        v = (size * normal(gen, n, 1, dim)).to(F16)
        want, _ = R.attention(q, k, v, [n], dim ** -0.5, d)
        got = gradients(ops, q, k, v, d, [n])
        near(got, want)
        # (each row by itself: its terms' sizes are its own; delta's error, from the rounded o, goes with the row's own o)
        for name in ("dk", "dq"):
            off, row = (got[name] - want[name]).norm(dim=2), want[name].norm(dim=2)
            keep = row > 2.0 ** -9                              # (rows whose results are normal numbers)
            assert float((off[keep] / row[keep]).max()) <= 4 * SIX, name


def test_nothing_to_scale(ops):
    """no gradients, no values, the smallest of both: noughts, and no NaN"""
    gen = torch.Generator().manual_seed(24)
    q, k, v, d = (normal(gen, 150, h, 64).to(F16) for h in (2, 1, 1, 2))
    for zero_v, zero_d in ((0.0, 1.0), (1.0, 0.0), (2.0 ** -24, 2.0 ** -24)):
        x, g = (torch.full_like(v, zero_v) if zero_v != 1.0 else v), (torch.full_like(d, zero_d) if zero_d != 1.0 else d)
        got = gradients(ops, q, k, x, g, [149, 1])
        assert bool((got["dq"] == 0).all()) and bool((got["dk"] == 0).all()) and bool(got["dv"].isfinite().all())


def test_gradients_that_are_not_finite_stay_in_their_sequence(ops):
    gen, n = torch.Generator().manual_seed(25), 227
    lengths = [100, 50, 77]
    q, k, v, d = (normal(gen, n, h, 64).to(F16).cuda() for h in (4, 2, 2, 4))
    packing = ops.Packing(lengths)
    o, lse = packing.attention(q, k, v)
    want = packing.attention_backward(d, q, k, v, o, lse)
    bad = d.clone()
    bad[100:150] = math.nan
    bad[120:130] = math.inf
    for a, b in zip(want, packing.attention_backward(bad, q, k, v, o, lse)):
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[150:], b[150:])
    # one query's: it reaches the keys that the query sees and its own dq, and no other key's
    bad = d.clone()
    bad[130, :2] = math.nan
    dq, dk, dv = packing.attention_backward(bad, q, k, v, o, lse)
    assert torch.equal(dq[:130], want[0][:130]) and torch.equal(dq[131:], want[0][131:]) and bool(dq[130, :2].isnan().all())
    for a, b in ((dk, want[1]), (dv, want[2])):
        assert torch.equal(a[:, 1], b[:, 1]) and bool(a[100:131, 0].isnan().all())


def test_probabilities_of_very_many_keys(ops):
    """queries that see 2^17 keys alike: probabilities of 2^-17 are rounded to as many bits as larger ones.  q = 0, so p = 1 / (i + 1); of dv, which
    is rounded twice, the last keys"""
    n, first = 200000, 1 << 17
    gen = torch.Generator().manual_seed(26)
    k, v = normal(gen, n, 1, 8).to(F16), normal(gen, n, 1, 8).to(F16)
    d = (2.0 ** 10 * normal(gen, n, 1, 8)).to(F16)
    got = gradients(ops, torch.zeros(n, 1, 8, dtype=F16), k, v, d, [n])["dv"]
    terms = d.double() / torch.arange(1, n + 1, dtype=torch.float64)[:, None, None]
    want = terms.flip(0).cumsum(0).flip(0)
    near({"dv": got[first:]}, {"dv": want[first:]}, ("dv",), 2 * 2.0 ** -11 + 2.0 ** -16)
