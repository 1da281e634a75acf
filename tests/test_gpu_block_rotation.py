"""The norms of queries and keys with the rotation by position, forward and backward, on the GPU against the definition in 64 bits: types, head layouts, even dims
of every kind, parts of heads, both orders of pairs, far positions, strides, added gradients, streams and graphs."""
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


def frequency(turning, base=10000.0):
    return base ** (-torch.arange(0, turning, 2, dtype=torch.float64) / max(1, turning))


def inputs(n, heads, kv_heads, dim, dtype, normed=True, seed=1):
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return 1.5 * torch.randn(*shape, generator=gen)
    v = {"q": normal(n, heads, dim).to(dtype), "k": normal(n, kv_heads, dim).to(dtype), "dq": normal(n, heads, dim).to(dtype), "dk": normal(n, kv_heads, dim).to(dtype)}
    v["wq"], v["wk"] = (1 + 0.3 * normal(dim), 1 + 0.3 * normal(dim)) if normed else (None, None)
    return v


def cuda(v):
    return {k: t.cuda() if t is not None else None for k, t in v.items()}


def wanted(v, position, f, eps, neighbours):
    return {name: R.rotation(v[name], position, f, v["w" + name], eps, neighbours, v["d" + name]) for name in ("q", "k")}


def check(ops, v, position, turning, neighbours=False, eps=1e-5, f=None, g=None):
    f = frequency(turning) if f is None else f
    g = cuda(v) if g is None else g
    at, fr = position.cuda(), f.cuda()
    args = (g["q"], g["k"], at, fr, g["wq"], g["wk"], eps, neighbours)
    q, k = ops.rotate(*args)
    dq, dk, dwq, dwk = ops.rotate_backward(g["dq"], g["dk"], *args)
    want = wanted(v, position, f, eps, neighbours)
    for name, got in (("q", (q, dq, dwq)), ("k", (k, dk, dwk))):
        for what, x, (value, bound) in zip(("result", "gradient", "gradient of w"), got, want[name]):
            if value is None:
                assert x is None
                continue
            assert x.dtype is (torch.float32 if what == "gradient of w" else v[name].dtype)
            R.close(x, value, bound, (what, name))


def positions(n, most=5000, seed=2, kind=torch.int64):
    return torch.randint(0, most, (n,), generator=torch.Generator().manual_seed(seed)).to(kind)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim, turning", [(128, 128), (128, 64), (64, 64), (64, 32), (256, 256), (96, 96), (40, 24), (80, 80), (8, 8)])
def test_heads(ops, dim, turning, dtype, normed, neighbours):
    check(ops, inputs(7, 6, 2, dim, dtype, normed, seed=dim), positions(7), turning, neighbours)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim, turning", [(2, 2), (2, 0), (4, 2), (6, 6), (6, 4), (10, 8), (12, 12), (16, 16), (16, 8), (18, 2), (24, 24), (32, 32), (48, 16), (50, 50), (66, 66), (72, 72),
                                          (100, 50), (112, 112), (120, 40), (126, 124), (128, 0), (128, 2), (128, 126), (136, 136), (160, 80), (192, 192), (200, 200), (224, 32), (254, 254),
                                          (254, 100), (256, 64), (256, 0), (256, 240), (128, 120), (80, 60), (256, 130), (256, 250), (22, 10), (20, 8), (40, 32), (18, 10)])
def test_dims_of_every_kind(ops, dim, turning, dtype):
    for neighbours in (False, True):
        check(ops, inputs(5, 3, 2, dim, dtype, True, seed=dim + turning), positions(5), turning, neighbours)


@pytest.mark.parametrize("n, heads, kv_heads", [(1, 1, 1), (1, 32, 8), (2, 5, 5), (3, 1, 7), (17, 40, 1), (64, 2, 1), (501, 3, 1), (1000, 8, 8), (3, 130, 65), (4111, 1, 1)])
def test_numbers_of_tokens_and_heads(ops, n, heads, kv_heads):
    check(ops, inputs(n, heads, kv_heads, 64, torch.bfloat16), positions(n, kind=torch.int32), 64)
    check(ops, inputs(n, heads, kv_heads, 24, torch.float32), positions(n), 12, True)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_far_positions(ops, kind):
    """angles of a million radians and more, and of positions before the first"""
    at = torch.tensor([0, 1, -1, 1 << 20, (1 << 20) + 1, (1 << 31) - 1, -(1 << 31), 999983], dtype=torch.int64)
    check(ops, inputs(8, 4, 2, 128, torch.float32), at.to(kind), 128)
    check(ops, inputs(8, 4, 2, 64, torch.bfloat16, False), at.to(kind), 64, True)


def test_other_frequencies(ops):
    """any numbers, not of a base alone"""
    f = torch.tensor([1.0, -0.37, 0.0, 3.5, 100.0, 1e-9], dtype=torch.float64)
    check(ops, inputs(9, 3, 3, 20, torch.float32), positions(9), 12, f=f)
    got = ops.frequencies(128, 500000.0).cpu()
    assert torch.allclose(got, 500000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128), rtol=1e-13, atol=0)


def test_position_nought_turns_nothing(ops):
    v = cuda(inputs(5, 4, 2, 64, torch.bfloat16, False))
    q, k = ops.rotate(v["q"], v["k"], torch.zeros(5, dtype=torch.int32, device="cuda"), frequency(64).cuda())
    assert torch.equal(q, v["q"]) and torch.equal(k, v["k"])


@pytest.mark.parametrize("neighbours", [False, True])
def test_channels_that_do_not_turn_stay_as_they_are(ops, neighbours):
    """bit by bit, infinities among them, and next to these too"""
    v = inputs(6, 2, 1, 64, torch.bfloat16, False)
    for n in ("q", "k", "dq", "dk"):
        v[n][1, 0, 40], v[n][2, 0, 63], v[n][3, 0, 16] = float("inf"), float("-inf"), float("nan")
    g = cuda(v)
    args = (g["q"], g["k"], positions(6).cuda(), frequency(16).cuda(), None, None, 1e-6, neighbours)
    for got, name in zip(ops.rotate(*args) + ops.rotate_backward(g["dq"], g["dk"], *args)[:2], ("q", "k", "dq", "dk")):
        assert torch.equal(got[..., 16:].view(torch.int16), g[name][..., 16:].view(torch.int16))
        assert bool(torch.isfinite(got[..., :16]).all())


def test_small_and_large_values(ops):
    """heads whose squares are subnormal numbers of 32 bits, with and without eps, and heads near the largest whose squares are numbers"""
    for size, eps in ((1e-20, 0.0), (3e-20, 0.0), (1e-19, 1e-37), (1e-12, 0.0), (1e18, 1e-6)):
        v = inputs(4, 2, 2, 64, torch.float32)
        for n in ("q", "k"):
            v[n] *= size
        g = cuda(v)
        at, f = positions(4), frequency(64)
        got = ops.rotate(g["q"], g["k"], at.cuda(), f.cuda(), g["wq"], g["wk"], eps)
        for x, n in zip(got, ("q", "k")):
            want, bound = R.rotation(v[n], at, f, v["w" + n], eps, False)[0]
            # squares of numbers around 2^-66 lose bits below 2^-149: 2^-17 of the mean of 64 of them, half that of its root
            R.close(x, want, bound + (2.0 ** -16 * R.both(want, 64, 64, False) if size < 1e-19 else 0.0), (n, size))


def test_heads_of_noughts(ops):
    """a head whose channels are all nought, of which eps is the whole norm"""
    v = inputs(4, 2, 2, 64, torch.float32)
    v["q"][1] = 0
    check(ops, v, positions(4), 64, eps=1e-3)


def test_values_that_are_no_numbers(ops):
    """stay in their heads"""
    v = inputs(40, 4, 2, 64, torch.bfloat16)
    clean = cuda(v)
    at, f = positions(40).cuda(), frequency(64).cuda()
    want = ops.rotate(clean["q"], clean["k"], at, f, clean["wq"], clean["wk"]) + ops.rotate_backward(clean["dq"], clean["dk"], clean["q"], clean["k"], at, f, clean["wq"], clean["wk"])[:2]
    bad = {k: t.clone() for k, t in clean.items()}
    bad["q"][7, 2, 5], bad["k"][0, 1, 63], bad["dq"][39, 3, 0], bad["dk"][20, 0, 33] = float("nan"), float("inf"), float("inf"), float("nan")
    got = ops.rotate(bad["q"], bad["k"], at, f, bad["wq"], bad["wk"]) + ops.rotate_backward(bad["dq"], bad["dk"], bad["q"], bad["k"], at, f, bad["wq"], bad["wk"])[:2]
    for x, y, touched in zip(got, want, ([(7, 2)], [(0, 1)], [(7, 2), (39, 3)], [(0, 1), (20, 0)])):
        for t, h in touched:
            assert not bool(torch.isfinite(x[t, h]).all())
            x[t, h] = y[t, h]
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim, odd", [(128, 0), (64, 0), (64, 1), (40, 3)])
def test_strides(ops, dim, odd, dtype):
    """parts of a joint projection, also one that starts and goes on at odd addresses; gradients into parts of a joint one; heads before tokens"""
    v = inputs(33, 6, 3, dim, dtype)
    wide = 12 * dim + odd

    def joint(q, k):
        t = torch.full((33, wide), float("nan"), dtype=dtype, device="cuda")
        a, b = t[:, odd:odd + 6 * dim].unflatten(1, (6, dim)), t[:, odd + 6 * dim:odd + 9 * dim].unflatten(1, (3, dim))
        a.copy_(q)
        b.copy_(k)
        return t, a, b
    _, q, k = joint(v["q"], v["k"])
    _, dq, dk = joint(v["dq"], v["dk"])
    g = dict(cuda(v), q=q, k=k, dq=dq, dk=dk)
    check(ops, v, positions(33), dim, g=g)
    t, a, b = joint(v["q"], v["k"])
    args = (q, k, positions(33).cuda(), frequency(dim).cuda(), g["wq"], g["wk"])
    want = ops.rotate_backward(dq, dk, *args)
    got = ops.rotate_backward(dq, dk, *args, out=(a, b))
    assert got[0] is a and torch.equal(a, want[0]) and torch.equal(b, want[1])
    assert bool(torch.isnan(t[:, :odd]).all()) and bool(torch.isnan(t[:, odd + 9 * dim:]).all())
    first = {n: t.transpose(0, 1).contiguous().transpose(0, 1) for n, t in (("q", g["q"]), ("k", g["k"]), ("dq", g["dq"]), ("dk", g["dk"]))}
    out = tuple(torch.empty(h, 33, dim, dtype=dtype, device="cuda").transpose(0, 1) for h in (6, 3))
    got = ops.rotate_backward(first["dq"], first["dk"], first["q"], first["k"], *args[2:], out=out)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    one = (g["q"][:, :1].expand(33, 6, dim), g["k"][:1].expand(33, 3, dim))              # (one head for all, one token for all)
    got = ops.rotate(*one, *args[2:])
    want = ops.rotate(one[0].contiguous(), one[1].contiguous(), *args[2:])
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_no_tokens(ops):
    q, k = (torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    at, w = torch.empty(0, dtype=torch.int64, device="cuda"), torch.ones(64, device="cuda")
    args = (q, k, at, frequency(64).cuda())
    assert [t.shape for t in ops.rotate(*args, w, w)] == [q.shape, k.shape]
    got = ops.rotate_backward(q, k, *args, w, w)
    assert all(torch.equal(t, torch.zeros(64, device="cuda")) for t in got[2:])
    kept = (torch.full((64,), 3.0, device="cuda"), torch.full((64,), 4.0, device="cuda"))
    ops.rotate_backward(q, k, *args, w, w, into=kept)
    assert bool((kept[0] == 3).all()) and bool((kept[1] == 4).all())
    assert ops.rotate_backward(q, k, *args)[2:] == (None, None)


def test_gradients_are_added(ops):
    v = cuda(inputs(300, 5, 2, 96, torch.bfloat16))
    args = (v["dq"], v["dk"], v["q"], v["k"], positions(300).cuda(), frequency(96).cuda(), v["wq"], v["wk"])
    once = ops.rotate_backward(*args)
    old = [torch.randn(96, device="cuda") for _ in range(2)]
    into = tuple(t.clone() for t in old)
    got = ops.rotate_backward(*args, into=into)
    assert got[2] is into[0] and got[3] is into[1]
    assert torch.equal(into[0], old[0] + once[2]) and torch.equal(into[1], old[1] + once[3])


def test_the_same_bits_twice(ops):
    v = cuda(inputs(3000, 6, 3, 64, torch.bfloat16))
    args = (v["dq"], v["dk"], v["q"], v["k"], positions(3000).cuda(), frequency(64).cuda(), v["wq"], v["wk"])
    assert all(torch.equal(a, b) for a, b in zip(ops.rotate_backward(*args), ops.rotate_backward(*args)))


def test_a_token_alone_is_what_it_is_among_others(ops):
    """the form for single tokens, and slices of a batch, bit by bit"""
    v = cuda(inputs(700, 8, 2, 128, torch.bfloat16))
    at, f = positions(700).cuda(), frequency(128).cuda()
    q, k = ops.rotate(v["q"], v["k"], at, f, v["wq"], v["wk"])
    for part in (slice(0, 1), slice(699, 700), slice(100, 103), slice(7, 300)):
        a, b = ops.rotate(v["q"][part], v["k"][part], at[part], f, v["wq"], v["wk"])
        assert torch.equal(a, q[part]) and torch.equal(b, k[part])


def test_more_heads_in_all_than_waves_of_a_launch(ops):
    """2^21 tokens of 32 + 8 heads: the first tokens, some and the last against the definition; only their gradients add to those of w"""
    n, dim = (1 << 21) + 3, 8
    part = torch.tensor([0, 1, 2, 5, 1 << 20, (1 << 20) + 1, n - 4, n - 2, n - 1])
    v, at, f = inputs(len(part), 32, 8, dim, torch.bfloat16), positions(len(part)), frequency(dim)
    g = {}
    for name, heads in (("q", 32), ("k", 8), ("dq", 32), ("dk", 8)):
        g[name] = torch.full((n, heads, dim), 0.0 if name[0] == "d" else 1.0, dtype=torch.bfloat16, device="cuda")
        g[name][part.cuda()] = v[name].cuda()
    where = torch.zeros(n, dtype=torch.int64)
    where[part] = at
    args = (g["q"], g["k"], where.cuda(), f.cuda(), v["wq"].cuda(), v["wk"].cuda(), 1e-5)
    out = ops.rotate(*args)
    grad = ops.rotate_backward(g["dq"], g["dk"], *args)
    want = wanted(v, at, f, 1e-5, False)
    for i, name in enumerate(("q", "k")):
        for what, x, (value, bound) in zip(("result", "gradient", "gradient of w"), (out[i][part.cuda()], grad[i][part.cuda()], grad[2 + i]), want[name]):
            R.close(x, value, bound, (what, name))
        assert int(grad[i].ne(0).any(-1).any(-1).sum()) <= len(part)


def test_strides_beyond_32_bits(ops):
    """tokens, and heads, further apart than 32 bits count, read and written there"""
    v = cuda(inputs(3, 2, 2, 64, torch.bfloat16))
    far, at, f = (1 << 32) + 8, positions(3).cuda(), frequency(64).cuda()
    big = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    want = ops.rotate(v["q"], v["k"], at, f, v["wq"], v["wk"])
    back = ops.rotate_backward(v["dq"], v["dk"], v["q"], v["k"], at, f, v["wq"], v["wk"])
    for strides in ((far, 64, 1), (64, far, 1)):
        q, k, dq, dk = (big.as_strided((3, 2, 64), strides, 256 * i) for i in range(4))
        q.copy_(v["q"])
        k.copy_(v["k"])
        got = ops.rotate(q, k, at, f, v["wq"], v["wk"])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        got = ops.rotate_backward(v["dq"], v["dk"], q, k, at, f, v["wq"], v["wk"], out=(dq, dk))
        assert got[0] is dq and all(torch.equal(a, b) for a, b in zip(got, back))


def test_a_graph_with_other_positions(ops):
    v = inputs(50, 4, 2, 64, torch.bfloat16)
    g, f = cuda(v), frequency(64).cuda()
    at = positions(50).cuda()

    def both():
        q, k = ops.rotate(g["q"], g["k"], at, f, g["wq"], g["wk"])
        return (q, k) + ops.rotate_backward(g["dq"], g["dk"], g["q"], g["k"], at, f, g["wq"], g["wk"])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for seed in range(4):
        at.copy_(positions(50, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, both()))                   # (eager work in between)


def test_refusals(ops):
    from paper_2311_15269_amd.binding import TesselError
    v = cuda(inputs(6, 4, 2, 64, torch.bfloat16))
    at, f = positions(6).cuda(), frequency(64).cuda()
    q, k, w = v["q"], v["k"], v["wq"]
    bad = [(q, k, at.float(), f), (q, k, at[:5], f), (q, k, at.cpu(), f), (q, k, at, f.float()), (q, k, at, frequency(66).cuda()), (q, k, at, f, w), (q, k, at, f, w, w[:60]),
           (q, k, at, f, w, w.bfloat16()), (q, k, at, f, w, w, -1.0), (q, k, at, f, w, w, float("nan")), (q[0], k, at, f), (q, k[:5], at, f), (q, k.float(), at, f), (q[..., :62], k, at, f),
           (q[..., :63], k[..., :63], at, f[:31]), (q.double(), k.double(), at, f), (q.transpose(1, 2), k.transpose(1, 2), at, f[:1]), (q[:, :0], k, at, f), (q, k[:, :0], at, f),
           (torch.zeros(6, 4, 258, device="cuda"), torch.zeros(6, 2, 258, device="cuda"), at, f), (q.clone().requires_grad_(), k, at, f), (q, k, at, f, w.clone().requires_grad_(), w)]
    for args in bad:
        with pytest.raises(TesselError):
            ops.rotate(*args)
    args = (v["dq"], v["dk"], q, k, at, f, w, w)
    both = torch.zeros(6, 4, 64, dtype=torch.bfloat16, device="cuda")
    for out in ((both[:, :1].expand(6, 4, 64), both[:, :2]), (both[:1].expand(6, 4, 64), both[:, :2]), (both, both), (both.as_strided((6, 4, 64), (64, 64, 1)), both[:, :2])):
        with pytest.raises(TesselError):
            ops.rotate_backward(*args, out=out)
    with pytest.raises(TesselError):
        ops.rotate_backward(v["dk"], v["dk"], *args[2:])
    with pytest.raises(TesselError):
        ops.rotate_backward(*args, into=(w, w[:60]))


def test_frequencies_that_require_a_gradient_are_refused(ops):
    """while torch records; they get none"""
    from paper_2311_15269_amd.binding import TesselError
    v = cuda(inputs(6, 4, 2, 64, torch.bfloat16))
    at, f = positions(6).cuda(), frequency(64).cuda().requires_grad_()
    for call in (lambda: ops.rotate(v["q"], v["k"], at, f), lambda: ops.rotate_backward(v["dq"], v["dk"], v["q"], v["k"], at, f, v["wq"], v["wk"])):
        with pytest.raises(TesselError):
            call()
        with torch.no_grad():
            call()


@pytest.mark.parametrize("neighbours", [False, True])
def test_positions_up_to_the_last_of_64_bits(ops, neighbours):
    """angles of 2^40 radians and more.  Of the angle there is what rounding its fraction of half a turn, the sine and cosine to 32 bits costs, 2^-21 with what the products add,
    and nothing that grows with it"""
    at = [0, 3, 1 << 40, -(1 << 45) - 1, (1 << 50) + 1, 1 << 53, (1 << 53) + 1, -(1 << 53) - 1, 12345678901234567, (1 << 62) + 3, (1 << 63) - 1, -(1 << 63)]
    f = torch.cat((frequency(56), torch.tensor([100.0, -0.37, 2.5, 1e-12], dtype=torch.float64)))
    v = inputs(len(at), 4, 2, 64, torch.float32, False)
    g, args = cuda(v), (torch.tensor(at).cuda(), f.cuda(), None, None, 1e-6, neighbours)
    angle = R.reduced_angles(at, f.tolist())
    got = dict(zip(("q", "k"), ops.rotate(g["q"], g["k"], *args))) | dict(zip(("dq", "dk"), ops.rotate_backward(g["dq"], g["dk"], g["q"], g["k"], *args)))
    for name, x in got.items():
        z = v[name].double()
        want = R.turned(z, -angle if name[0] == "d" else angle, 64, 64, neighbours)
        R.close(x, want, R.H * want.abs() * (1 + 1e-3) + (2.0 ** -21 + 6 * R.H) * R.both(z, 64, 64, neighbours), name)
