"""Activation checkpoints in 8 bits on the GPU: stored numbers exactly as defined, the gated activation and its gradients and the
weight gradient against the definition in 64 bits, at ragged sizes, extreme values, strides, streams and graphs."""
import math

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import block_ops
    return block_ops


def rows(n, c, dtype, seed, by=1.0):
    gen = torch.Generator().manual_seed(seed)
    spread = torch.exp(torch.randn(c, generator=gen))
    return (by * spread * torch.randn(n, c, generator=gen)).to(dtype)


def check_store(ops, x):
    whole, exponent = R.held(x)
    c = ops.checkpoint(x.cuda())
    n, channels = x.shape
    bad = exponent == -1000
    assert torch.equal(c.exponents.cpu().long(), torch.where(bad, torch.zeros_like(exponent), exponent + 127))
    keep = ~bad.repeat_interleave(64, 1)[:, :channels]
    assert torch.equal(c.values[:, :channels].cpu().double()[keep], whole[keep])
    y, want = ops.restore(c), R.values(whole, exponent)
    assert y.dtype == x.dtype and y.shape == x.shape
    assert torch.equal(y.cpu().double()[keep], want[keep]) and bool(y.cpu()[~keep].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, c", [(1, 1), (1, 64), (3, 63), (5, 65), (2, 127), (7, 200), (33, 129), (1, 2000), (40, 8)])
def test_store_and_restore(ops, n, c, dtype):
    check_store(ops, rows(n, c, dtype, n + c))


@pytest.mark.parametrize("dtype", TYPES)
def test_values_at_the_ends_of_the_type(ops, dtype):
    info = torch.finfo(dtype)
    x = rows(12, 64, dtype, 3)
    x[0] = 0
    x[1, 5] = info.max
    x[2, 5] = -info.max
    x[3] = info.tiny
    x[4] = 0
    x[4, 0] = info.smallest_normal / 4                              # below the normal numbers
    x[5, 9] = math.inf
    x[6, 9] = math.nan
    x[7, 1], x[7, 2] = -math.inf, math.nan
    x[8, 0] = 127.5
    x[9, 0] = 127.0
    x[10, 0] = 255.0
    x[11] = torch.arange(64).to(dtype) + 0.5                        # ties: to the even number
    x[11, 0] = 100.0
    check_store(ops, x)


def test_error_of_a_checkpoint(ops):
    """half a step, which is at most 1/127.5 of the group's largest value, and a checkpoint of a checkpoint is the same"""
    for dtype in TYPES:
        x = rows(50, 256, dtype, 8).cuda()
        y = ops.restore(ops.checkpoint(x))
        most = x.double().abs().view(50, 4, 64).amax(2, keepdim=True)
        assert bool(((x - y).double().abs().view(50, 4, 64) <= most / 127.5 * (1 + 1e-12)).all())
        assert torch.equal(ops.restore(ops.checkpoint(y)), y)


def near(got, want, dtype, size, what):
    """rounded once, and 4e-6 of the product of the factors' sizes for 32-bit arithmetic: the exponential of arguments up to 30 (30 x
    2^-24 and its own 2^-22), and a dozen operations"""
    off = (got.double().cpu() - want).abs() - R.U[dtype] * want.abs() - R.TINY[dtype] - 4e-6 * size
    assert float(off.max()) <= 0.0, (what, float(off.max()))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, c", [(1, 1), (3, 64), (5, 100), (17, 333), (2, 1024)])
def test_gated(ops, n, c, dtype, act):
    g, u, da = rows(n, c, dtype, 1, 0.7).clamp(-20, 20), rows(n, c, dtype, 2), rows(n, c, dtype, 3)
    a, kg, ku = ops.gated(g.cuda(), u.cuda(), act)
    near(a, R.act(act, g.double()) * u.double(), dtype, (1 + g.double().abs()) * u.double().abs(), "a")
    hg, hu = R.values(*R.held(g)), R.values(*R.held(u))
    assert torch.equal(ops.restore(kg).cpu().double(), hg) and torch.equal(ops.restore(ku).cpu().double(), hu)
    dg, du, again = ops.gated_backward(da.cuda(), kg, ku, act, with_output=True)
    x, y = hg.clone().requires_grad_(), hu.clone().requires_grad_()
    wg, wu = torch.autograd.grad(R.act(act, x) * y, [x, y], da.double())
    d = da.double().abs()
    near(dg, wg, dtype, d * hu.abs() * (1 + hg.abs()) * (1 + hg.abs()), "dg")
    near(du, wu, dtype, d * (1 + hg.abs()), "du")
    near(again, R.act(act, hg) * hu, dtype, (1 + hg.abs()) * hu.abs(), "a of the checkpoints")
    two = ops.gated_backward(da.cuda(), kg, ku, act)
    assert len(two) == 2 and torch.equal(two[0], dg) and torch.equal(two[1], du)


def test_gated_of_large_values(ops):
    """arguments at which the exponential leaves 32 bits: nought or the argument itself"""
    for act in ("silu", "gelu"):
        g = torch.tensor([[-300.0, -100.0, 100.0, 300.0, 0.0]], device="cuda")
        u = torch.ones_like(g)
        a, kg, ku = ops.gated(g, u, act)
        assert float((a.cpu() - torch.tensor([[0.0, 0.0, 100.0, 300.0, 0.0]])).abs().max()) <= 1e-4
        dg, du = ops.gated_backward(u, kg, ku, act)
        assert float((dg.cpu() - torch.tensor([[0.0, 0.0, 1.0, 1.0, 0.5]])).abs().max()) <= 1e-4 and bool(du.isfinite().all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gated_where_powers_of_the_argument_leave_32_bits(ops, dtype):
    for act in ("silu", "gelu"):
        g = torch.tensor([1e12, 1e13, 1.8e19, 2e19, 1e25, 1e38], device="cuda")[:, None]
        g = torch.cat([g, -g]).to(dtype)
        u = torch.ones_like(g)
        a, kg, ku = ops.gated(g, u, act)
        dg, du, again = ops.gated_backward(u, kg, ku, act, with_output=True)
        kept = ops.restore(kg)
        assert torch.equal(a, g.clamp(min=0)) and torch.equal(again, kept.clamp(min=0)) and torch.equal(du, again)
        assert torch.equal(dg, (g > 0).to(dtype))


def check_weight(ops, n, m, c, dtype, seed=1, into=None):
    dy, x = rows(n, m, dtype, seed), rows(n, c, dtype, seed + 1)
    k = ops.checkpoint(x.cuda())
    held = ops.restore(k).double().cpu()
    want = dy.double().T @ held
    start = None if into is None else torch.full((m, c), into, device="cuda")
    got = ops.weight_gradient(dy.cuda(), k, start)
    if into is not None:
        assert got is start
        want = want + into
    # products are exact in 32 bits; n of them are added one after another or in parts: n 2^-24 of their sizes at worst
    bound = (n + 16) * 2.0 ** -24 * (dy.double().abs().T @ held.abs() + abs(into or 0.0))
    off = (got.double().cpu() - want).abs() - bound
    assert float(off.max()) <= 0.0, (n, m, c, dtype, float(off.max()))


@pytest.mark.parametrize("dtype", TYPES[:2])
@pytest.mark.parametrize("n, m, c", [(1, 1, 1), (1, 8, 64), (63, 64, 64), (64, 128, 128), (65, 129, 127), (200, 7, 300), (300, 300, 9), (257, 136, 200),
                                     (1500, 130, 260), (5000, 33, 70), (700, 256, 512)])
def test_weight_gradient(ops, n, m, c, dtype):
    check_weight(ops, n, m, c, dtype)
    check_weight(ops, n, m, c, dtype, into=1.5)


@pytest.mark.parametrize("m", [5, 7, 8, 9, 104, 131])
@pytest.mark.parametrize("n", [2, 64, 127, 128, 129, 191, 193, 256, 257, 513, 640, 1025])
def test_weight_gradient_where_tiles_of_tokens_end(ops, n, m):
    """outputs of less than a chunk, of whole chunks and of others; tokens that leave the second group of waves nothing, less or as much"""
    check_weight(ops, n, m, 70, torch.bfloat16)
    check_weight(ops, n, m, 70, torch.float16, into=-0.5)


@pytest.mark.parametrize("n, m, c", [(1, 4096, 2048), (130, 4096, 2050), (130, 4095, 2048), (64, 2051, 4001)])
def test_weight_gradient_by_large_tiles(ops, n, m, c):
    check_weight(ops, n, m, c, torch.bfloat16)
    check_weight(ops, n, m, c, torch.bfloat16, into=0.25)


@pytest.mark.parametrize("m", [2048, 2050])
def test_weight_gradient_by_large_tiles_in_splits(ops, m):
    check_weight(ops, 5300, m, 2048, torch.float16, into=1.0)


@pytest.mark.parametrize("m", [6, 64, 77])
@pytest.mark.parametrize("token", [0, 63, 99])
def test_weight_gradient_of_gradients_that_are_not_finite(ops, m, token):
    """an output's infinity or NaN reaches its own row and no other"""
    dy, x = rows(100, m, torch.bfloat16, 1), rows(100, 200, torch.bfloat16, 2)
    k = ops.checkpoint(x.cuda())
    want = ops.weight_gradient(dy.cuda(), k)
    dy[token, m - 1], dy[token, 2] = math.inf, math.nan
    got = ops.weight_gradient(dy.cuda(), k)
    held = ops.restore(k)[token].float()
    assert bool(got[2].isnan().all())
    signs = torch.where(held == 0, torch.nan, held.sign() * math.inf)
    assert torch.equal(got[m - 1].nan_to_num(7.0, 8.0, 9.0), signs.nan_to_num(7.0, 8.0, 9.0))
    others = [i for i in range(m) if i not in (2, m - 1)]
    assert torch.equal(got[others], want[others])


def test_weight_gradient_of_no_tokens(ops):
    k = ops.checkpoint(torch.empty(0, 100, dtype=torch.bfloat16, device="cuda"))
    dy = torch.empty(0, 30, dtype=torch.bfloat16, device="cuda")
    assert bool((ops.weight_gradient(dy, k) == 0).all())
    kept = torch.full((30, 100), 2.0, device="cuda")
    assert bool((ops.weight_gradient(dy, k, kept) == 2.0).all())


def test_weight_gradient_of_values_that_are_not_finite(ops):
    """a group that is not finite gives NaN in its columns and nowhere else"""
    dy, x = rows(100, 70, torch.bfloat16, 1).cuda(), rows(100, 200, torch.bfloat16, 2).cuda()
    want = ops.weight_gradient(dy, ops.checkpoint(x))
    x[40, 70] = math.inf
    got = ops.weight_gradient(dy, ops.checkpoint(x))
    assert bool(got[:, 64:128].isnan().all())
    assert torch.equal(got[:, :64], want[:, :64]) and torch.equal(got[:, 128:], want[:, 128:])


def test_strides_and_offsets(ops):
    for dtype in TYPES:
        x = rows(30, 150, dtype, 4).cuda()
        room = torch.empty(30, 157, dtype=dtype, device="cuda")
        wide = room[:, 3:153]
        wide.copy_(x)
        a, b = ops.checkpoint(x), ops.checkpoint(wide)
        assert torch.equal(a.exponents, b.exponents) and torch.equal(ops.restore(a), ops.restore(b))
        one, two = ops.gated(x, x), ops.gated(wide, wide)
        assert torch.equal(one[0], two[0])
        for p, q in zip(ops.gated_backward(x, *one[1:]), ops.gated_backward(wide, *two[1:])):
            assert torch.equal(p, q)
        if dtype != torch.float32:
            sums = torch.zeros(150, 160, device="cuda")[:, 5:155]
            want = ops.weight_gradient(x, a)
            assert torch.equal(want, ops.weight_gradient(wide, b)) and torch.equal(want, ops.weight_gradient(wide, b, sums))


def test_streams_graphs_and_repeats(ops):
    g, u, da = (rows(400, 700, torch.bfloat16, s).cuda() for s in (1, 2, 3))

    def all_of_it():
        a, kg, ku = ops.gated(g, u)
        dg, du = ops.gated_backward(da, kg, ku)
        return a, dg, du, ops.restore(ops.checkpoint(g)), ops.weight_gradient(da, kg)
    want = all_of_it()
    for a, b in zip(want, all_of_it()):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_of_it()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for turn in range(3):
        g.mul_(0.75)
        for t in got:
            t.fill_(9.0)
        want = all_of_it()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b), turn


def test_refusals(ops):
    from paper_2311_15269_amd.binding import TesselError
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    k = ops.checkpoint(x)
    for call in (lambda: ops.checkpoint(x.double()), lambda: ops.checkpoint(x.t()), lambda: ops.checkpoint(x[0]), lambda: ops.gated(x, x[:3]),
                 lambda: ops.gated(x, x.half()), lambda: ops.gated(x, x, "relu"), lambda: ops.gated_backward(x[:2], k, k),
                 lambda: ops.gated_backward(x, k, ops.checkpoint(x[:2])), lambda: ops.weight_gradient(x[:3], k), lambda: ops.weight_gradient(x.half(), k),
                 lambda: ops.weight_gradient(x.float(), ops.checkpoint(x.float())), lambda: ops.weight_gradient(x, k, torch.zeros(64, 63, device="cuda")),
                 lambda: ops.weight_gradient(x, k, torch.zeros(64, 64, device="cuda").half())):
        with pytest.raises(TesselError):
            call()
