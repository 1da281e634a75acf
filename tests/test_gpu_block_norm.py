"""The norms around a block with gate and residual scale, forward and backward, on the GPU against the definition in 64 bits:
every shape of row the kernels tell apart, odd sizes, types, gates, strides, added gradients, streams and graphs."""
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


def inputs(n, c, dtype, gate, post, seed=1):
    gen = torch.Generator().manual_seed(seed)

    def rows(by=1.0):
        return (by * torch.randn(n, c, generator=gen)).to(dtype)
    v = {"x": rows(), "y": rows(2.0), "dr": rows(), "dh": rows(), "pre": 1 + 0.3 * torch.randn(c, generator=gen),
         "post": 1 + 0.3 * torch.randn(c, generator=gen) if post else None, "gate": None}
    if gate == "channel":
        v["gate"] = torch.randn(c, generator=gen)
    elif gate == "token":
        v["gate"] = rows()
    return v


def close(got, want, dtype, size, what):
    """rounded once (u of the value), and 1e-5 of `size` for the sums in 32 bits: rows of 16384 squares in a tree of at most 16 + 8 + 10
    additions, and columns of some hundred terms, stay below 2^-17 of the sum of their terms' sizes"""
    got = got.double().cpu()
    off = (got - want).abs() - R.U[dtype] * want.abs() - R.TINY[dtype] - 1e-5 * size
    assert float(off.max()) <= 0.0, (what, float(off.max()))


def check(ops, n, c, dtype, gate, post, scale=0.75, eps=1e-5, seed=1):
    v = inputs(n, c, dtype, gate, post, seed)
    want = R.norm(v["x"], v["y"], v["pre"], v["post"], v["gate"], scale, eps, v["dr"], v["dh"])
    g = {k: t.cuda() if t is not None else None for k, t in v.items()}
    r, h, stats = ops.residual_norm(g["x"], g["y"], g["pre"], g["post"], g["gate"], scale, eps)
    got = ops.residual_norm_backward(g["dr"], g["dh"], g["x"], g["y"], stats, g["pre"], g["post"], g["gate"], scale)
    # sizes of the terms that the values are sums of
    x, y, dr, dh, pre = (v[k].double().abs() for k in ("x", "y", "dr", "dh", "pre"))
    over_y = 1 / torch.sqrt((y * y).mean(1, keepdim=True) + eps) if post else 1.0
    w = v["post"].double().abs() if post else 1.0
    gt = v["gate"].double().abs() if gate != "none" else 1.0
    u = y * over_y * w
    rs = scale * x + gt * u
    over_r = 1 / torch.sqrt((want["r"] ** 2).mean(1, keepdim=True) + eps)
    rn = rs * over_r
    drs = dr + over_r * (dh * pre + rn * (dh * pre * rn).mean(1, keepdim=True))
    dus = drs * gt
    yn = y * over_y
    dys = over_y * (dus * w + yn * (dus * w * yn).mean(1, keepdim=True)) if post else dus
    close(r, want["r"], dtype, rs, "r")
    close(h, want["h"], dtype, rn * pre, "h")
    close(got[0], want["dx"], dtype, scale * drs, "dx")
    close(got[1], want["dy"], dtype, dys, "dy")
    close(got[2], want["dpre"], torch.float32, (dh * rn).sum(0), "dpre")
    if post:
        close(got[3], want["dpost"], torch.float32, (dus * yn).sum(0), "dpost")
    else:
        assert got[3] is None
    if gate == "channel":
        close(got[4], want["dgate"], torch.float32, (drs * u).sum(0), "dgate")
    elif gate == "token":
        close(got[4], want["dgate"], dtype, drs * u, "dgate")
    else:
        assert got[4] is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [1, 7, 8, 9, 64, 511, 512, 513, 1000, 1024, 1025, 2048, 2056, 4095, 4096, 4097, 8192, 8200, 16383, 16384])
def test_rows_of_every_shape(ops, c, dtype):
    check(ops, 5, c, dtype, "channel", True, seed=c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("post", [True, False])
def test_gates_and_norms(ops, dtype, gate, post):
    check(ops, 9, 300, dtype, gate, post)
    check(ops, 6, 2500, dtype, gate, post)


@pytest.mark.parametrize("n, c", [(1, 64), (3, 5000), (600, 40), (2100, 130), (1030, 2049), (4500, 16)])
def test_numbers_of_tokens(ops, n, c):
    check(ops, n, c, torch.bfloat16, "channel", True)


def test_no_tokens(ops):
    x = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(96, device="cuda")
    r, h, stats = ops.residual_norm(x, x, w, w, w)
    assert r.shape == h.shape == (0, 96)
    got = ops.residual_norm_backward(x, x, x, x, stats, w, w, w)
    for g in got[2:]:
        assert torch.equal(g, torch.zeros(96, device="cuda"))
    kept = [torch.full((96,), 3.0, device="cuda") for _ in range(3)]
    ops.residual_norm_backward(x, x, x, x, stats, w, w, w, into=kept)
    assert all(bool((g == 3.0).all()) for g in kept)


def test_gradients_are_added(ops):
    v = {k: t.cuda() for k, t in inputs(70, 1300, torch.bfloat16, "channel", True).items()}
    r, h, stats = ops.residual_norm(v["x"], v["y"], v["pre"], v["post"], v["gate"])
    args = (v["dr"], v["dh"], v["x"], v["y"], stats, v["pre"], v["post"], v["gate"])
    one = ops.residual_norm_backward(*args)
    kept = [torch.full((1300,), 2.0, device="cuda") for _ in range(3)]
    two = ops.residual_norm_backward(*args, into=kept)
    for a, b, c in zip(one[2:], two[2:], kept):
        assert b is c
        assert float((b - 2.0 - a).abs().max()) <= 2.0 ** -22 * (2.0 + float(a.abs().max())) * 4     # (added first, 9 additions)


def test_rows_of_nought_and_values_that_are_not_finite(ops):
    """a row of zeros is divided by sqrt(eps); a row with NaN or infinity leaves its neighbours alone"""
    for c in (300, 3000):
        v = {k: t.cuda() for k, t in inputs(6, c, torch.bfloat16, "channel", True).items()}
        v["x"][1] = 0
        v["y"][1] = 0
        clean = ops.residual_norm(v["x"], v["y"], v["pre"], v["post"], v["gate"])
        assert bool((clean[0][1] == 0).all()) and bool((clean[1][1] == 0).all()) and bool(clean[2].isfinite().all())
        bad = v["y"].clone()
        bad[3, 5] = float("nan")
        bad[4, 7] = float("inf")
        r, h, _ = ops.residual_norm(v["x"], bad, v["pre"], v["post"], v["gate"])
        for row in (0, 1, 2, 5):
            assert torch.equal(r[row], clean[0][row]) and torch.equal(h[row], clean[1][row])
        assert bool(h[3].isnan().all()) and bool(h[4].isnan().any())


def test_strides_and_offsets(ops):
    for dtype in TYPES:
        for c in (65, 2064):
            v = {k: t.cuda() for k, t in inputs(40, c, dtype, "token", True).items()}
            want = ops.residual_norm(v["x"], v["y"], v["pre"], v["post"], v["gate"])
            back = ops.residual_norm_backward(v["dr"], v["dh"], v["x"], v["y"], want[2], v["pre"], v["post"], v["gate"])
            wide = {}
            for i, k in enumerate(("x", "y", "gate", "dr", "dh")):
                room = torch.empty(40, c + 3 + i, dtype=dtype, device="cuda")
                wide[k] = room[:, 1 + i % 3:1 + i % 3 + c]
                wide[k].copy_(v[k])
            got = ops.residual_norm(wide["x"], wide["y"], v["pre"], v["post"], wide["gate"])
            for a, b in zip(got, want):
                assert torch.equal(a, b)
            again = ops.residual_norm_backward(wide["dr"], wide["dh"], wide["x"], wide["y"], want[2], v["pre"], v["post"], wide["gate"])
            for a, b in zip(again, back):
                assert torch.equal(a, b)
    x = torch.randn(1, 512, device="cuda").expand(20, 512)          # the same row for every token
    w = torch.ones(512, device="cuda")
    r, h, _ = ops.residual_norm(x, x, w)
    one, two, _ = ops.residual_norm(x.contiguous(), x.contiguous(), w)
    assert torch.equal(r, one) and torch.equal(h, two)


def test_streams_graphs_and_repeats(ops):
    v = {k: t.cuda() for k, t in inputs(900, 1100, torch.bfloat16, "channel", True).items()}

    def both():
        r, h, stats = ops.residual_norm(v["x"], v["y"], v["pre"], v["post"], v["gate"])
        return (r, h, *ops.residual_norm_backward(v["dr"], v["dh"], v["x"], v["y"], stats, v["pre"], v["post"], v["gate"]))
    want = both()
    for a, b in zip(want, both()):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for turn in range(3):
        v["y"].mul_(0.5)
        for t in got:
            t.fill_(9.0)
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b), turn


def test_refusals(ops):
    from paper_2311_15269_amd.binding import TesselError
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for bad in ((x, x[:3], w), (x, x.half(), w), (x, x, w[:32]), (x, x, w.half()), (x, x, w, w[:3]), (x, x, w, w, x[:2]), (x.double(), x.double(), w),
                (x.t(), x.t(), torch.ones(4, device="cuda")), (torch.zeros(1, 20000, device="cuda"),) * 2 + (torch.ones(20000, device="cuda"),)):
        with pytest.raises(TesselError):
            ops.residual_norm(*bad)
    r, h, stats = ops.residual_norm(x, x, w)
    for bad in ((r[:2], h, x, x, stats, w), (r, h, x, x, stats[:1], w), (r, h, x, x, stats.t(), w)):
        with pytest.raises(TesselError):
            ops.residual_norm_backward(*bad)
