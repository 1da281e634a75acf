"""A transformer stage in the order of a searched schedule: its gradients against torch's differentiation of the same stage in 64 bits, the
schedule's order against one micro-batch after the other, and what 8-bit checkpoints save."""
import pytest
import torch

pytestmark = pytest.mark.gpu
LENGTHS = [100, 1, 27]


@pytest.fixture(scope="module")
def stage():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import stage
    return stage


def plain(s, x, h):
    """the stage from its definition in 64 bits on the CPU: (r, h, dict of leaves)"""
    leaf = {k: w.double().cpu().requires_grad_() for k, w in s.weights.items()}
    norms = [{k: v.double().cpu().requires_grad_() for k, v in n.items()} for n in s.norms]
    x, h = x.double().cpu().requires_grad_(), h.double().cpu().requires_grad_()

    def norm(z, w):
        return w * z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-6)

    def around(i, z, y):
        r = s.scale * z + norms[i]["gate"] * norm(y, norms[i]["post"])
        return r, norm(r, norms[i]["pre"])
    n = x.shape[0]
    qkv = (h @ leaf["qkv"].T).view(n, -1, s.dim)
    heads = []
    for i in range(s.heads):
        j = s.heads + i * s.kv_heads // s.heads
        q, k, v = qkv[:, i], qkv[:, j], qkv[:, j + s.kv_heads]
        rows, begin = [], 0
        for length in LENGTHS:
            at = slice(begin, begin + length)
            seen = torch.ones(length, length, dtype=torch.bool).tril()
            rows.append(torch.softmax((q[at] @ k[at].T / s.dim ** 0.5).masked_fill(~seen, -torch.inf), 1) @ v[at])
            begin += length
        heads.append(torch.cat(rows))
    r, hr = around(0, x, torch.cat(heads, 1) @ leaf["out"].T)
    z = (torch.nn.functional.silu(hr @ leaf["gate"].T) * (hr @ leaf["up"].T)) @ leaf["down"].T
    r, h2 = around(1, r, z)
    return r, h2, leaf, norms, x, h


def off(got, want):
    want = want.detach()
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("small", [True, False])
def test_gradients_of_a_stage(stage, small):
    """A checkpoint's error is at most half a step, a step at most 1/63.75 of the group's largest value, which is some 2.5 times the root
    mean square of 64 normal numbers: 1.2 % of it as a root mean square of a uniform error.  16-bit values are rounded to 0.2 % a dozen times on the way.
    Together below 5 % of a gradient's norm."""
    (s,), (packing,), (x,), (h,) = stage.make(1, 1, LENGTHS, 128, 4, 2, 256, small, seed=5)
    r, hr = s.forward(0, packing, x, h)
    gen = torch.Generator().manual_seed(6)
    dr, dh = (torch.randn(r.shape, generator=gen).bfloat16() for _ in range(2))
    dx, dhx = s.backward(0, dr.cuda(), dh.cuda())
    wr, wh, leaf, norms, lx, lh = plain(s, x, h)
    assert off(r, wr) < 0.02 and off(hr, wh) < 0.02
    torch.autograd.backward([wr, wh], [dr.double(), dh.double()])
    assert off(dx, lx.grad) < 0.05 and off(dhx, lh.grad) < 0.05
    for k, w in leaf.items():
        assert off(s.gradients[k], w.grad) < 0.05, k
    for n, g in zip(norms, s.norm_gradients):
        for k in n:
            assert off(g[k], n[k].grad) < 0.05, k
    assert not s.kept


def test_the_order_of_a_schedule_changes_nothing(stage):
    sizes = (3, 6, LENGTHS, 128, 4, 2, 256, True)
    stages, packings, xs, hs = stage.make(*sizes)
    found, done, operations = stage.plan(3, (1.0, 2.1), 3, 9, 6, max_nr=3)
    assert found["best_nr"] >= 1 and done["makespan"] > 0
    blocks = [op[1] for op in operations if op[0] == 0]
    assert sorted(blocks) == list(range(6 * 6))
    dr = torch.randn_like(xs[0])
    got = stage.run(stages, packings, xs, hs, lambda mu, r, h: (dr, h), operations)
    again, packings, xs, hs = stage.make(*sizes)
    want = stage.run(again, packings, xs, hs, lambda mu, r, h: (dr, h), stage.in_turn(3, 6))
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for s, t in zip(stages, again):
        for k in s.gradients:
            assert torch.equal(s.gradients[k], t.gradients[k]), k
        for g, h in zip(s.norm_gradients, t.norm_gradients):
            for k in g:
                assert torch.equal(g[k], h[k]), k


def test_what_checkpoints_save(stage):
    """the same cap holds more micro-batches, and the search reaches its lower bound"""
    kept = []
    for small in (False, True):
        (s,), (packing,), (x,), (h,) = stage.make(1, 1, LENGTHS, 128, 4, 2, 512, small)
        s.forward(0, packing, x, h)
        kept.append(-(-s.kept_bytes(0) // x.numel()))
    assert kept[1] < 0.75 * kept[0]
    cap = 3 * kept[0]
    wide, narrow = (stage.plan(4, (1.0, 2.0), m, cap, 12)[0] for m in kept)
    assert narrow["inflights"] > wide["inflights"]
    assert narrow["best_period"] / narrow["best_nr"] < wide["best_period"] / wide["best_nr"]
