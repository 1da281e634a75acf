"""Dropout whose mask is never stored, on the GPU against its definition bit by bit: types, odd sizes, strides, numbers that pass 32 bits, values that are
no numbers, the backward pass as the same call, streams and graphs that draw anew."""
import pytest
import torch

from tests import entry_reference as R

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import block_ops
    return block_ops


def rows(n, c, dtype, seed=1):
    return torch.randn(n, c, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, c", [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (1, 4096), (130, 1003), (33, 64), (700, 12), (2, 16385)])
def test_every_value(ops, dtype, n, c):
    x = rows(n, c, dtype)
    for rate, seed, number in ((0.1, 5, 0), (0.5, (1 << 64) - 1, (1 << 64) - 1), (0.9999999, 1 << 40, 3 << 31)):
        got = ops.dropout(x.cuda(), ops.Dropout(rate, seed, number))
        assert torch.equal(got.cpu(), R.dropped(x, rate, seed, number)), (rate, seed, number)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_dropout(ops, dtype):
    x = rows(17, 130, dtype)
    assert torch.equal(ops.dropout(x.cuda(), ops.Dropout(0.0, 5)).cpu(), x)


def test_strides(ops):
    x = rows(60, 100, torch.bfloat16)
    g = x.cuda()
    for part in ((slice(None, None, 3), slice(3, 80)), (slice(5, 6), slice(None)), (slice(None), slice(1, 2))):
        want = R.dropped(x[part].contiguous(), 0.3, 9, 1)
        assert torch.equal(ops.dropout(g[part], ops.Dropout(0.3, 9, 1)).cpu(), want)
    wide = g[:1].expand(40, 100)                                    # (one row, read forty times, with a mask for each)
    assert torch.equal(ops.dropout(wide, ops.Dropout(0.3, 9, 1)).cpu(), R.dropped(x[:1].expand(40, 100).contiguous(), 0.3, 9, 1))


def test_no_tokens(ops):
    assert ops.dropout(torch.empty(0, 8, device="cuda"), ops.Dropout(0.5, 1)).shape == (0, 8)


def test_what_is_dropped_is_zero_whatever_it_was(ops):
    x = torch.full((50, 40), float("nan"))
    x[:, ::2] = float("inf")
    got = ops.dropout(x.cuda(), ops.Dropout(0.5, 3, 4)).cpu()
    keep, _ = R.kept(50, 40, 0.5, 3, 4)
    assert bool((got[~keep] == 0).all()) and bool(torch.isnan(got[:, 1::2][keep[:, 1::2]]).all()) and bool(torch.isinf(got[:, ::2][keep[:, ::2]]).all())


def test_gradient(ops):
    """sum(dropout(x) dy) changes with x by dropout(dy)"""
    x, dy = rows(31, 77, torch.float32, 1).cuda(), rows(31, 77, torch.float32, 2).cuda()
    drop = ops.Dropout(0.4, 8, 9)
    h = (torch.randint(0, 3, (31, 77), generator=torch.Generator().manual_seed(3)) - 1).float().cuda()      # (x + h is not rounded further than x)
    # |x| < 8 and |x + h| < 8: their own rounding, the two products' and the difference's are below 2^-19 for each value
    change = ((ops.dropout(x + h, drop).double() - ops.dropout(x, drop).double()) * dy.double()).sum()
    want = (h.double() * ops.dropout(dy, drop).double()).sum()
    assert abs(float(change - want)) < 31 * 77 * 2.0 ** -19 * 5


def test_steps_on_the_gpu(ops):
    """a step is added to the number, into its upper half too"""
    x = rows(40, 100, torch.float16)
    for number, step in ((0, 0), (7, 5), ((1 << 32) - 1, 1), (3, (1 << 33) + 1), ((1 << 64) - 1, 2)):
        s = torch.tensor([step], device="cuda")
        got = ops.dropout(x.cuda(), ops.Dropout(0.2, 6, number, s))
        assert torch.equal(got.cpu(), R.dropped(x, 0.2, 6, number + step))


def test_a_graph_draws_anew(ops):
    x = rows(64, 300, torch.bfloat16)
    g, step = x.cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = ops.Dropout(0.25, 4, 100, step)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ops.dropout(g, drop)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.dropout(g, drop)
        dx = ops.dropout(y, drop)
        step += 1
    step.zero_()
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = R.dropped(x, 0.25, 4, 100 + k)
        assert torch.equal(y.cpu(), want) and torch.equal(dx.cpu(), R.dropped(want, 0.25, 4, 100 + k))
        assert torch.equal(ops.dropout(g, ops.Dropout(0.25, 4, 7)).cpu(), R.dropped(x, 0.25, 4, 7))      # (eager work in between)


def test_on_another_stream(ops):
    x = rows(512, 2000, torch.bfloat16)
    stream = torch.cuda.Stream()
    g = x.cuda()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        y = ops.dropout(g, ops.Dropout(0.5, 2))
    stream.synchronize()
    assert torch.equal(y.cpu(), R.dropped(x, 0.5, 2, 0))


def test_many_rows(ops):
    """more values than 32 bits count, the last rows of them"""
    n, c = (1 << 31) // 1000 + 50, 1000
    x = torch.zeros(n, c, dtype=torch.float16, device="cuda")
    x[-40:] = rows(40, c, torch.float16).cuda()
    y = ops.dropout(x, ops.Dropout(0.5, 2, 3))
    assert not bool(y[:1000].any())
    for t in (n - 40, n - 1):
        want = [R.philox([k // 4, t, 3, 0], [2, 0])[k % 4] >= 1 << 31 for k in range(c)]
        assert torch.equal(y[t].cpu(), torch.where(torch.tensor(want), x[t].cpu() * 2, 0))


def test_refusals(ops):
    from paper_2311_15269_amd.binding import TesselError
    for args in ((1.0, 1), (-0.1, 1), (float("nan"), 1), (0.5, -1), (0.5, 1 << 64), (0.5, 1, -1), (0.5, 1, 0, torch.zeros(1, dtype=torch.int64)),
                 (0.5, 1, 0, torch.zeros(2, dtype=torch.int64, device="cuda")), (0.5, 1, 0, torch.zeros(1, device="cuda"))):
        with pytest.raises(TesselError):
            ops.Dropout(*args)
    drop, x = ops.Dropout(0.5, 1), torch.zeros(4, 8, device="cuda")
    for bad in (x[0], x.double(), x.t()[::1], x.cpu(), x.clone().requires_grad_()):
        with pytest.raises(TesselError):
            ops.dropout(bad, drop)
    with torch.no_grad():
        ops.dropout(x.clone().requires_grad_(), drop)
