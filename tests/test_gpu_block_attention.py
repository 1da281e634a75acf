"""Packed causal attention on the GPU against the definition in 64 bits, element by element within derived bounds
(tests/block_reference.py): lengths from none to several tiles, heads that share keys, every width, strides, tokens of no
sequence, what no query may see, streams and graphs."""
import math

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import block_ops
    return block_ops


def inputs(n, heads, kv_heads, dim, dtype, seed, by=1.0):
    gen = torch.Generator().manual_seed(seed)

    def make(h):
        return (by * torch.randn(n, h, dim, generator=gen)).to(dtype)
    return make(heads), make(kv_heads), make(kv_heads), make(heads)


def near(got, want, bound, what):
    got = got.double().cpu()
    same = torch.isinf(want) & (got == want)
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    assert not bool(torch.isnan(off).any()) and float(off.max() if off.numel() else 0.0) <= 0.0, (what, float(off.max()))


def check(ops, lengths, heads, kv_heads, dim, dtype, seed=1, padding=0, scale=None, by=1.0):
    n = sum(lengths) + padding
    q, k, v, d = inputs(n, heads, kv_heads, dim, dtype, seed, by)
    want, bound = R.attention(q, k, v, lengths, 1 / math.sqrt(dim) if scale is None else scale, d)
    packing = ops.Packing(lengths, n)
    gq, gk, gv, gd = (t.cuda() for t in (q, k, v, d))
    o, lse = packing.attention(gq, gk, gv, scale)
    dq, dk, dv = packing.attention_backward(gd, gq, gk, gv, o, lse, scale)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        near(got, want[name], bound[name], (name, lengths, heads, kv_heads, dim, dtype))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths", [[1], [2], [31], [32], [33], [63], [64], [65], [127], [128], [129], [255], [257], [300]])
def test_one_sequence(ops, lengths, dtype):
    check(ops, lengths, 2, 1, 64, dtype)


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 64, 72, 80, 96, 120, 128])
def test_widths(ops, dim):
    check(ops, [70, 130], 2, 2, dim, BF16, seed=dim)
    check(ops, [70, 130], 2, 1, dim, F16, seed=dim)


@pytest.mark.parametrize("heads, kv_heads", [(1, 1), (3, 1), (6, 3), (5, 5), (8, 8), (8, 1), (8, 2), (16, 4), (24, 8), (16, 16)])
def test_head_layouts(ops, heads, kv_heads):
    check(ops, [150, 20], heads, kv_heads, 64, BF16, seed=heads)


@pytest.mark.parametrize("lengths, padding", [([], 7), ([0], 3), ([0, 0, 1, 0], 0), ([5, 0, 0, 129, 1, 64, 0], 0), ([1] * 70, 130), ([40, 3], 257),
                                              ([129, 128, 127, 1, 2, 3], 1)])
def test_packings(ops, lengths, padding):
    check(ops, lengths, 4, 2, 128, BF16, padding=padding)
    check(ops, lengths, 4, 2, 64, F16, padding=padding)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_several_tiles_of_wide_heads(ops, dtype):
    check(ops, [700, 1, 385], 4, 2, 128, dtype)


@pytest.mark.parametrize("lengths, heads, kv_heads, dim, dtype", [([1500], 1, 1, 64, BF16), ([1500], 2, 1, 128, F16), ([1030, 5, 200], 2, 2, 128, BF16),
                                                                  ([1025, 0, 640], 4, 1, 40, F16), ([600, 600], 3, 1, 96, BF16), ([64 * 17 + 1], 2, 1, 128, BF16)])
def test_few_heads_over_long_sequences(ops, lengths, heads, kv_heads, dim, dtype):
    """work split over keys and queries, and joined: tiles with fewer steps than splits, heads that share keys, tokens of none"""
    check(ops, lengths, heads, kv_heads, dim, dtype, padding=9)


@pytest.mark.parametrize("dtype, by", [(BF16, 0.01), (BF16, 3.0), (F16, 0.01), (F16, 3.0)])
def test_sizes_of_values(ops, dtype, by):
    """scores all alike, and scores that leave one key a row"""
    check(ops, [200, 90], 2, 1, 64, dtype, by=by)


def test_scale(ops):
    check(ops, [100], 2, 1, 64, BF16, scale=0.03)
    check(ops, [100], 2, 1, 64, BF16, scale=1.0)


def test_small_gradients_in_half_precision(ops):
    """gradients a thousand times smaller: the scores' gradients keep their digits, so that only the results' own rounding differs"""
    q, k, v, d = inputs(200, 2, 2, 64, F16, 5)
    d[:] = torch.where(d.abs() < 2.0 ** -4, torch.zeros_like(d), d)           # (exact after scaling)
    packing = ops.Packing([200])
    o, lse = packing.attention(q.cuda(), k.cuda(), v.cuda())
    want = packing.attention_backward(d.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)
    got = packing.attention_backward((d * 2.0 ** -10).cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)
    for a, b in zip(want[:2], got[:2]):
        a, b = a.double() * 2.0 ** -10, b.double()
        assert bool(((a - b).abs() <= 2.0 ** -11 * a.abs() + 2.0 ** -24).all())


def test_sequences_and_heads_keep_their_own_scale(ops):
    """in half precision the gradients of one sequence, and of the heads on one key, do not depend on the sizes of others'"""
    q, k, v, d = (t.cuda() for t in inputs(260, 4, 2, 64, F16, 6))
    packing = ops.Packing([100, 160])
    o, lse = packing.attention(q, k, v)
    want = packing.attention_backward(d, q, k, v, o, lse)
    far = d.clone()
    far[:100] *= 500.0
    far[:, 2:] = math.inf
    got = packing.attention_backward(far, q, k, v, o, lse)
    for a, b, heads in zip(want, got, (2, 1, 1)):
        assert torch.equal(a[100:, :heads], b[100:, :heads])


@pytest.mark.parametrize("token", [0, 31, 127, 128, 2047, 2048, 2499])
def test_the_largest_gradient_may_be_anywhere(ops, token):
    """in half precision: one query's gradient 2^14 times the others', which those of the scores must not leave the type's range for.  Rounding
    probabilities, gradients of the scores and results: 2^-11 each of the largest, six of them at most"""
    q, k, v, d = inputs(2500, 2, 1, 64, F16, 7)
    d = d * 2.0 ** -4
    d[token] *= 2.0 ** 14
    want, _ = R.attention(q, k, v, [2500], 0.125, d)
    packing = ops.Packing([2500])
    gq, gk, gv, gd = (t.cuda() for t in (q, k, v, d))
    o, lse = packing.attention(gq, gk, gv)
    for name, got in zip(("dq", "dk", "dv"), packing.attention_backward(gd, gq, gk, gv, o, lse)):
        got = got.double().cpu()
        assert bool(got.isfinite().all()), name
        assert float((got - want[name]).norm()) <= 6 * 2.0 ** -11 * float(want[name].norm()), name


def test_strided_views(ops):
    """one tensor of all projections, heads before tokens, keys shared through a stride of nought"""
    lengths, n = [90, 41], 131
    q, k, v, d = inputs(n, 4, 2, 64, BF16, 9)
    packing = ops.Packing(lengths)
    want = packing.attention(q.cuda(), k.cuda(), v.cuda())
    back = packing.attention_backward(d.cuda(), q.cuda(), k.cuda(), v.cuda(), *want)
    both = torch.cat([q, k, v], 1).cuda()
    a, b, c = both[:, :4], both[:, 4:6], both[:, 6:]
    turned = [t.cuda().transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v, d)]
    for x, y, z, g in ((a, b, c, d.cuda()), turned):
        o, lse = packing.attention(x, y, z)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        for got, ref in zip(packing.attention_backward(g, x, y, z, o, lse), back):
            assert torch.equal(got, ref)
    one = k[:, :1].cuda()
    wide = one.expand(n, 4, 64)
    o, lse = packing.attention(q.cuda(), wide, wide)
    ref, _ = packing.attention(q.cuda(), one, one)
    assert torch.equal(o, ref)
    dq, dk, dv = packing.attention_backward(d.cuda(), q.cuda(), wide, wide, o, lse)
    want, bound = R.attention(q, wide.cpu(), wide.cpu(), lengths, 0.125, d)
    near(dk, want["dk"], bound["dk"], "dk of a broadcast key")
    near(dv, want["dv"], bound["dv"], "dv of a broadcast value")


def test_sequences_do_not_see_each_other(ops):
    """infinities and NaN in one sequence, and in tokens of none, change nothing elsewhere"""
    lengths, padding = [100, 50, 77], 30
    n = sum(lengths) + padding
    for dtype in (BF16, F16):
        q, k, v, d = (t.cuda() for t in inputs(n, 4, 2, 64, dtype, 11))
        packing = ops.Packing(lengths, n)
        o, lse = packing.attention(q, k, v)
        back = packing.attention_backward(d, q, k, v, o, lse)
        bad = [t.clone() for t in (q, k, v, d)]
        for t in bad:
            t[100:150] = math.nan
            t[120:130] = math.inf
            t[227:] = math.nan
        o2, lse2 = packing.attention(*bad[:3])
        if dtype == F16:
            bad[3][100:150] = d[100:150]                        # (its scale is taken from all gradients of sequences)
        back2 = packing.attention_backward(bad[3], *bad[:3], o2, lse2)
        for a, b in zip((o, *back), (o2, *back2)):
            assert torch.equal(a[:100], b[:100]) and torch.equal(a[150:], b[150:])
            assert bool((b[227:] == 0).all())
        assert torch.equal(lse[:, :100], lse2[:, :100]) and torch.equal(lse[:, 150:], lse2[:, 150:])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128])
def test_queries_do_not_see_later_tokens(ops, dtype, dim):
    """infinities and NaN in a sequence's keys and values leave the tokens before them alone, and reach those behind"""
    n = 300
    q, k, v, _ = (t.cuda() for t in inputs(n, 2, 1, dim, dtype, 16, 0.5))
    packing = ops.Packing([n])
    o, lse = packing.attention(q, k, v)
    for at in (3, 70, 127, 150, 191, 260):
        bad_k, bad_v = k.clone(), v.clone()
        bad_v[at, 0, 5] = math.inf
        bad_v[at + 10:at + 12, 0, 7] = math.nan
        bad_v[at + 20, 0, 5] = -math.inf
        bad_k[at + 30] = math.nan
        o2, lse2 = packing.attention(q, bad_k, bad_v)
        assert torch.equal(o[:at], o2[:at]) and torch.equal(lse[:, :at + 30], lse2[:, :at + 30])
        rest = [c for c in range(dim) if c not in (5, 7)]
        assert bool((o2[at:at + 20, :, 5] == math.inf).all()) and bool(o2[at + 20:at + 30, :, 5].isnan().all())
        assert torch.equal(o[at:at + 10, :, 7], o2[at:at + 10, :, 7]) and bool(o2[at + 10:at + 30, :, 7].isnan().all())
        assert torch.equal(o[at:at + 30][:, :, rest], o2[at:at + 30][:, :, rest])
        assert bool(o2[at + 30:].isnan().all()) and bool(lse2[:, at + 30:].isnan().all())


def test_repeats_are_equal(ops):
    q, k, v, d = (t.cuda() for t in inputs(900, 8, 2, 128, BF16, 12))
    packing = ops.Packing([500, 3, 397])
    o, lse = packing.attention(q, k, v)
    back = packing.attention_backward(d, q, k, v, o, lse)
    for _ in range(3):
        o2, lse2 = packing.attention(q, k, v)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        for a, b in zip(back, packing.attention_backward(d, q, k, v, o2, lse2)):
            assert torch.equal(a, b)


def test_another_stream_and_a_graph(ops):
    q, k, v, d = (t.cuda() for t in inputs(300, 4, 4, 64, BF16, 13))
    packing = ops.Packing([200, 100])
    want = packing.attention(q, k, v)
    back = packing.attention_backward(d, q, k, v, *want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, lse = packing.attention(q, k, v)
        got = packing.attention_backward(d, q, k, v, o, lse)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o, want[0])
    for a, b in zip(got, back):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = packing.attention(q, k, v)
        got = packing.attention_backward(d, q, k, v, o, lse)
    for turn in range(3):
        for t in (o, *got):
            t.fill_(7.0)
        q.mul_(0.9)
        want = packing.attention(q, k, v)
        back = packing.attention_backward(d, q, k, v, *want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]), turn
        for a, b in zip(got, back):
            assert torch.equal(a, b), turn


def test_more_than_two_to_the_31_elements(ops):
    """heads of a strided tensor whose last tokens lie behind 2^31 elements"""
    n, stride = 300, 1 << 23
    room = torch.empty(n * stride, dtype=BF16, device="cuda")
    q, k, v, d = (t.cuda() for t in inputs(n, 2, 1, 64, BF16, 14))
    wide = room.as_strided((n, 2, 64), (stride, 64, 1))
    wide.copy_(q)
    packing = ops.Packing([n])
    o, lse = packing.attention(q, k, v)
    o2, lse2 = packing.attention(wide, k, v)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(packing.attention_backward(d, q, k, v, o, lse), packing.attention_backward(d, wide, k, v, o, lse)):
        assert torch.equal(a, b)


def test_refusals(ops):
    from paper_2311_15269_amd.binding import TesselError
    q, k, v, d = (t.cuda() for t in inputs(10, 4, 2, 64, BF16, 15))
    packing = ops.Packing([10])
    for bad in ((q[:9], k, v), (q, k[:, :1], v), (q, k.half(), v), (q.float(), k.float(), v.float()), (q, k, v[..., :32]),
                (q[..., ::2], k[..., ::2], v[..., ::2]), (q[:, :3], k, v)):
        with pytest.raises(TesselError):
            packing.attention(*bad)
    o, lse = packing.attention(q, k, v)
    for bad in ((d[:9], q, k, v, o, lse), (d, q, k, v, o[:, :2], lse), (d, q, k, v, o, lse.t()), (d, q, k, v, o, lse.double())):
        with pytest.raises(TesselError):
            packing.attention_backward(*bad)
