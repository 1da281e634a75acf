"""The embedding of a shard of the vocabulary and its gradient, on the GPU against the definition in 64 bits: types, odd sizes, tokens of other shards and of none,
every token the same, tables of one row to millions, added gradients, dropout, strides, streams and graphs."""
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


def inputs(n, rows, c, dtype, seed=1, low=0, high=None):
    gen = torch.Generator().manual_seed(seed)
    token = torch.randint(low, rows if high is None else high, (n,), generator=gen)
    return token, torch.randn(rows, c, generator=gen).to(dtype), torch.randn(n, c, generator=gen).to(dtype)


def check(ops, token, table, d, scale=1.5, first=0, drop=None):
    """forward, and the gradient written and added"""
    D = ops.Dropout(*drop) if drop else None
    at, rows = token.cuda(), table.shape[0]
    out = ops.embed(at, table.cuda(), scale, first, D)
    assert out.dtype is table.dtype and torch.equal(out.cpu(), R.embedding(token, table, scale, first, drop))
    want, bound = R.embedding_gradient(d, token, rows, scale, first, drop)
    got = ops.embed_backward(d.cuda(), at, rows, scale, first, D)
    R.close(got, want, bound, "dtable")
    old = torch.randn(want.shape, generator=torch.Generator().manual_seed(9))
    into = old.cuda()
    assert ops.embed_backward(d.cuda(), at, rows, scale, first, D, into=into) is into
    R.close(into, want + old.double(), 2 * bound + R.H * (want.abs() + old.double().abs()) * 1.01, "added")
    seen = torch.zeros(rows, dtype=torch.bool)
    seen[(token - first)[(token >= first) & (token < first + rows)]] = True
    assert torch.equal(into.cpu()[~seen], old[~seen]) and not bool(got.cpu()[~seen].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [1, 2, 7, 8, 9, 63, 64, 100, 1003, 2048, 2056, 4100, 9000])
def test_channels(ops, c, dtype):
    check(ops, *inputs(70, 23, c, dtype, seed=c))


@pytest.mark.parametrize("n, rows", [(1, 1), (1, 1000), (2, 2), (63, 5), (64, 64), (65, 300), (1000, 1), (1000, 3), (1023, 257), (1025, 256), (4096, 255), (4097, 5000),
                                     (9000, 70000), (20000, 40), (3000, 1100000), (40, 1 << 21)])
def test_tokens_and_rows(ops, n, rows):
    check(ops, *inputs(n, rows, 24 if rows < 100000 else 8, torch.bfloat16, seed=n + rows))


@pytest.mark.parametrize("n", [2, 4, 64, 65, 255, 256, 257, 300, 511, 512, 513])
@pytest.mark.parametrize("c", [3, 520, 4096, 4104])
def test_few_tokens(ops, n, c):
    """batches of one launch and of three, tokens of waves that have none in common and some"""
    token, table, d = inputs(n, 40, c, torch.bfloat16, seed=n + c, low=-2)
    check(ops, token, table, d)
    if c < 4000:
        check(ops, torch.full((n,), 39), table, d, drop=(0.3, 4, 5))


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
@pytest.mark.parametrize("first", [0, 37, 1000])
def test_shards(ops, first, kind):
    """tokens of the shard, of those before and behind it, and of none"""
    token, table, d = inputs(500, 50, 40, torch.float16, seed=first, low=-20, high=1100)
    token[::3] = first + token[::3].abs() % 50
    token[5], token[6], token[7], token[8] = first - 1, first, first + 49, first + 50
    check(ops, token.to(kind), table, d, first=first)


def test_the_ends_of_whole_numbers(ops):
    token, table, d = inputs(12, 9, 16, torch.bfloat16)
    for kind, far in ((torch.int64, 1 << 62), (torch.int32, 0)):
        t = token.to(kind) + far
        t[0], t[1], t[2] = torch.iinfo(kind).min, torch.iinfo(kind).max, -1
        check(ops, t, table, d, first=far)


def test_a_shard_without_tokens(ops):
    token, table, d = inputs(300, 20, 48, torch.bfloat16, low=100, high=200)
    check(ops, token, table, d)
    check(ops, torch.full((300,), -1), table, d)


def test_no_tokens(ops):
    table = torch.ones(10, 16, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert ops.embed(none, table).shape == (0, 16)
    empty = torch.empty(0, 16, device="cuda")
    assert torch.equal(ops.embed_backward(empty, none, 10), torch.zeros(10, 16, device="cuda"))
    assert torch.equal(ops.embed_backward(empty, none, 10, into=table.clone()), table)


@pytest.mark.parametrize("n, c", [(700, 64), (5000, 136), (30000, 40)])
def test_one_token_nearly_everywhere(ops, n, c):
    """padding that counts: nearly all of a batch is one token, whose gradient is one long sum"""
    token, table, d = inputs(n, 900, c, torch.bfloat16, seed=n)
    token[torch.rand(n, generator=torch.Generator().manual_seed(2)) < 0.9] = 513
    check(ops, token, table, d)
    check(ops, torch.full((n,), 899), table, d)


def test_runs_of_every_length(ops):
    """sums of 1, 2, .. 200 rows, in order and mixed"""
    token = torch.repeat_interleave(torch.arange(1, 201), torch.arange(1, 201))
    _, table, d = inputs(token.shape[0], 201, 32, torch.float16)
    check(ops, token, table, d)
    check(ops, token[torch.randperm(token.shape[0], generator=torch.Generator().manual_seed(5))], table, d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [8, 61, 1000])
def test_dropout_in_the_same_pass(ops, c, dtype):
    token, table, d = inputs(333, 40, c, dtype, low=-3)
    check(ops, token, table, d, drop=(0.3, 12345678901234567, (1 << 32) - 5))
    # the same as a dropout of its own behind it, but for the rounding between the two
    one = ops.Dropout(0.5, 1, 2)
    got = ops.embed(token.cuda(), table.cuda(), 2.0, 0, one)
    assert torch.equal(got, ops.dropout(ops.embed(token.cuda(), table.cuda(), 2.0), one))      # (powers of two)


def test_values_that_are_no_numbers(ops):
    """reach the tokens and the rows that they are of; rows of d_out whose token is not of the shard are not read"""
    token, table, d = inputs(600, 30, 40, torch.float32, low=-10, high=40)
    table[4, 3], table[5, :] = float("nan"), float("inf")
    out = ops.embed(token.cuda(), table.cuda(), 1.0).cpu()
    want = R.embedding(token, table, 1.0, 0)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.isinf(out), torch.isinf(want))
    d[(token < 0) | (token >= 30)] = float("nan")
    clean, _ = R.embedding_gradient(torch.nan_to_num(d), token, 30, 1.0, 0)
    where = int((token == 7).nonzero()[0])
    d[where, 11] = float("inf")
    got = ops.embed_backward(d.cuda(), token.cuda(), 30).cpu()
    assert got[7, 11] == float("inf")
    got[7, 11] = clean[7, 11]
    assert bool(torch.isfinite(got).all())


def test_strides(ops):
    token, table, d = inputs(200, 50, 96, torch.bfloat16)
    big = torch.zeros(60, 200, dtype=torch.bfloat16)
    big[3:53, 5:101] = table
    out = ops.embed(token.cuda(), big.cuda()[3:53, 5:101])
    assert torch.equal(out.cpu(), R.embedding(token, table, 1.0, 0))
    wide = torch.full((200, 131), float("nan"), dtype=torch.bfloat16)
    wide[:, 7:103] = d
    sums = torch.full((50, 130), 3.0, device="cuda")
    ops.embed_backward(wide.cuda()[:, 7:103], token.cuda(), 50, into=sums[:, 1:97])
    want, bound = R.embedding_gradient(d, token, 50, 1.0, 0)
    R.close(sums[:, 1:97], want + 3.0, 2 * bound + R.H * (want.abs() + 3.0) * 1.01, "strided sums")
    assert bool((sums[:, :1] == 3.0).all()) and bool((sums[:, 97:] == 3.0).all())
    one = d[:1].cuda().expand(200, 96)
    R.close(ops.embed_backward(one, token.cuda(), 50), *R.embedding_gradient(d[:1].expand(200, 96), token, 50, 1.0, 0), "one row for all")


def test_the_same_bits_twice(ops):
    token, table, d = inputs(20000, 300, 72, torch.bfloat16)
    a, b = (ops.embed_backward(d.cuda(), token.cuda(), 300, 0.3) for _ in range(2))
    assert torch.equal(a, b)


def test_the_gradient_is_that_of_the_lookup(ops):
    """sum(embed(table) d) changes with the table by embed_backward(d)"""
    token, table, d = inputs(400, 30, 20, torch.float32, low=-5, high=35)
    h = torch.zeros(30, 20)
    h[::2, ::3] = 0.5
    for drop in (None, ops.Dropout(0.5, 3, 4)):
        change = (ops.embed(token.cuda(), h.cuda(), 2.0, 0, drop).double() * d.cuda().double()).sum()         # (linear)
        grad = ops.embed_backward(d.cuda(), token.cuda(), 30, 2.0, 0, drop).double().cpu()
        # powers of two but for the sums, each a bound of its own
        _, bound = R.embedding_gradient(d, token, 30, 2.0, 0, (0.5, 3, 4) if drop else None)
        assert abs(float(change) - float((grad * h.double()).sum())) <= float((bound * h.double()).sum()) + 1e-9


def test_a_graph_with_other_tokens(ops):
    token, table, d = inputs(3000, 700, 64, torch.bfloat16)
    at, dev, grad = token.cuda(), table.cuda(), torch.zeros(700, 64, device="cuda")
    dd = d.cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ops.embed(at, dev)
        ops.embed_backward(dd, at, 700)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.embed(at, dev, 0.5)
        written = ops.embed_backward(dd, at, 700, 0.5)
        ops.embed_backward(dd, at, 700, 0.5, into=grad)
    grad.zero_()
    total = torch.zeros(700, 64, dtype=torch.float64)
    slack = torch.zeros(700, 64, dtype=torch.float64)
    for k in range(4):
        token = inputs(3000, 700 if k % 2 else 3, 1, torch.bfloat16, seed=50 + k, low=-2)[0]
        at.copy_(token)
        graph.replay()
        torch.cuda.synchronize()
        want, bound = R.embedding_gradient(d, token, 700, 0.5, 0)
        assert torch.equal(out.cpu(), R.embedding(token, table, 0.5, 0))
        R.close(written, want, bound, "replay %d" % k)
        assert torch.equal(written, ops.embed_backward(dd, at, 700, 0.5))           # (eager work in between)
        total += want
        slack += 2 * bound + R.H * total.abs() * 1.01 + R.H * slack
        R.close(grad, total, slack, "sums of replay %d" % k)


def test_two_streams_at_once(ops):
    token, table, d = inputs(8000, 5000, 256, torch.bfloat16)
    other = token.flip(0)
    g = [t.cuda() for t in (token, other, d)]
    want = [ops.embed_backward(g[2], t, 5000) for t in g[:2]]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(ops.embed_backward(g[2], g[k], 5000))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[k]) for k in range(2) for x in got[k])


def test_tables_beyond_32_bits(ops):
    """more values than 32 bits count"""
    rows, c = 1 << 23, 264
    token = torch.tensor([0, rows - 1, 5, rows - 1, rows // 2, rows])
    table = torch.zeros(rows, c, dtype=torch.bfloat16, device="cuda")
    d = torch.randn(6, c, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    for n in token[:5].tolist():
        table[n] = n % 250
    out = ops.embed(token.cuda(), table)
    assert [float(x) for x in out[:, c - 1]] == [0.0, float((rows - 1) % 250), 5.0, float((rows - 1) % 250), float(rows // 2 % 250), 0.0]
    del table, out
    for into in (None, torch.zeros(rows, c, device="cuda")):
        got = ops.embed_backward(d.cuda(), token.cuda(), rows, into=into)
        x = d.double()
        for n, want in ((0, x[0]), (rows - 1, x[1] + x[3]), (5, x[2]), (rows // 2, x[4]), (7, 0 * x[0]), (rows - 2, 0 * x[0])):
            assert torch.allclose(got[n].double().cpu(), want, rtol=0, atol=0 if n != rows - 1 else 2.0 ** -21)     # (one sum of two, below 8)
        assert int((got[::4099].abs().amax(1) > 0).sum()) == 1
        del got


def test_refusals(ops):
    from paper_2311_15269_amd.binding import TesselError
    token, table, d = (t.cuda() for t in inputs(6, 5, 16, torch.bfloat16))
    bad = [lambda: ops.embed(token.float(), table), lambda: ops.embed(token.view(2, 3), table), lambda: ops.embed(token.cpu(), table), lambda: ops.embed(token, table.double()),
           lambda: ops.embed(token, table.t()), lambda: ops.embed(token, table, float("inf")), lambda: ops.embed(token, table, first=-1), lambda: ops.embed(token, table[:0]),
           lambda: ops.embed(torch.stack((token, token), 1)[:, 0], table), lambda: ops.embed(token, table.clone().requires_grad_()), lambda: ops.embed(token, table[0]),
           lambda: ops.embed_backward(d, token[:5], 5), lambda: ops.embed_backward(d, token, 0), lambda: ops.embed_backward(d, token, (1 << 24) + 1, into=None),
           lambda: ops.embed_backward(d, token, 5, into=torch.zeros(5, 16)), lambda: ops.embed_backward(d, token, 5, into=torch.zeros(5, 16, device="cuda").bfloat16()),
           lambda: ops.embed_backward(d, token, 5, into=torch.zeros(16, 5, device="cuda").t()), lambda: ops.embed_backward(d, token, 5, into=torch.zeros(4, 16, device="cuda"))]
    for call in bad:
        with pytest.raises(TesselError):
            call()


@pytest.mark.parametrize("n", [16383, 16384, 16385, 32768, 40001, 65536, 65537, 100003])
@pytest.mark.parametrize("hot", [0.0, 0.2, 0.97])
def test_long_batches(ops, n, hot):
    """batches of several tiles, of which a bucket's places fit its list, and do not"""
    gen = torch.Generator().manual_seed(n)
    token = torch.randint(-3, 1000, (n,), generator=gen)
    token[torch.rand(n, generator=gen) < hot] = 300
    d = torch.randn(n, 8, generator=gen).to(torch.bfloat16)
    for kind in (torch.int64, torch.int32):
        got = ops.embed_backward(d.cuda(), token.to(kind).cuda(), 990)
        R.close(got, *R.embedding_gradient(d, token, 990, 1.0, 0), "dtable")


def test_more_pieces_of_zeros_than_workgroups(ops):
    """2.2 million rows of 2050 channels, a workgroup a row and more than 2^20 of them, for few tokens and for many"""
    rows, c = 2200000, 2050
    for n in (5, 600):
        token = torch.randint(0, rows, (n,), generator=torch.Generator().manual_seed(n))
        token[0], token[1] = 0, rows - 1
        got = torch.full((rows, c), float("nan"), device="cuda")
        del got                                                     # (the memory that the call below is likely to get)
        got = ops.embed_backward(torch.ones(n, c, dtype=torch.bfloat16, device="cuda"), token.cuda(), rows)
        assert torch.equal(got.sum(1, dtype=torch.float64).cpu(), c * torch.bincount(token, minlength=rows).double())
        del got
