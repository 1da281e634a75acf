"""The operators between the tokens and the attention together, as a stage runs them behind an embedding: against torch's differentiation of the same in 64 bits, in the
order of a schedule, over shards of the vocabulary, and as one captured training step."""
import pytest
import torch

from tests import entry_reference as R

pytestmark = pytest.mark.gpu
LENGTHS = [100, 1, 27]
TURNING, RATE, SEED = 16, 0.2, 5


@pytest.fixture(scope="module")
def stage():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import stage
    return stage


def mask(n, c, number):
    keep, by = R.kept(n, c, RATE, SEED, number)
    return keep.double() * float(by)


def plain(s, entry, tokens, mu):
    """an entry and a stage from their definitions in 64 bits on the CPU: (r, h, dict of leaves)"""
    leaf = {k: w.double().cpu().requires_grad_() for k, w in s.weights.items()}
    norms = [{k: v.double().cpu().requires_grad_() for k, v in n.items()} for n in s.norms]
    heads = [w.double().cpu().requires_grad_() for w in s.head_norms]
    table, pre = torch.cat(entry.tables).double().cpu().requires_grad_(), entry.pre.double().cpu().requires_grad_()
    n, c = tokens.shape[0], table.shape[1]
    position = torch.cat([torch.arange(m) for m in LENGTHS]).double()
    angle = position[:, None] * 10000.0 ** (-torch.arange(0, TURNING, 2, dtype=torch.float64) / TURNING)

    def norm(z, w):
        return w * z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-6)

    def around(i, z, y):
        r = s.scale * z + norms[i]["gate"] * norm(y, norms[i]["post"])
        return r, norm(r, norms[i]["pre"])
    x = mask(n, c, mu << 32 | 0xFFFFFFFF) * c ** 0.5 * table[tokens.cpu()]
    h = norm(x, pre)
    qkv = (h @ leaf["qkv"].T).view(n, -1, s.dim)
    q, k = (R.turned(norm(z, w), angle, s.dim, TURNING, False) for z, w in ((qkv[:, :s.heads], heads[0]), (qkv[:, s.heads:s.heads + s.kv_heads], heads[1])))
    rows, begin = [], 0
    for length in LENGTHS:
        at = slice(begin, begin + length)
        seen = torch.ones(length, length, dtype=torch.bool).tril()
        v = qkv[at, s.heads + s.kv_heads:]
        rows.append(torch.cat([torch.softmax((q[at, i] @ k[at, i * s.kv_heads // s.heads].T / s.dim ** 0.5).masked_fill(~seen, -torch.inf), 1) @ v[:, i * s.kv_heads // s.heads]
                               for i in range(s.heads)], 1))
        begin += length
    r, hr = around(0, x, mask(n, c, mu << 32) * (torch.cat(rows) @ leaf["out"].T))
    z = mask(n, c, mu << 32 | 1) * ((torch.nn.functional.silu(hr @ leaf["gate"].T) * (hr @ leaf["up"].T)) @ leaf["down"].T)
    r, h2 = around(1, r, z)
    leaf.update(table=table, pre=pre, wq=heads[0], wk=heads[1])
    return r, h2, leaf, norms


def off(got, want):
    want = want.detach()
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("small", [True, False])
def test_gradients_of_an_entry_and_a_stage(stage, small):
    """bounds as for a stage alone: checkpoints of 8 bits 1.2 % of an input's root mean square, roundings to 16 bits 0.2 % each, together below 5 %"""
    (s,), (packing,), _, _ = stage.make(1, 1, LENGTHS, 128, 4, 2, 256, small, seed=SEED, turning=TURNING, rate=RATE)
    entry, (tokens,) = stage.make_entry(1, LENGTHS, 128, 300, 3, seed=SEED, rate=RATE)
    for w in s.head_norms:
        w.copy_(1 + 0.3 * torch.randn(w.shape, generator=torch.Generator().manual_seed(3)))
    mu = 7
    x, h = entry.forward(mu, tokens)
    r, hr = s.forward(mu, packing, x, h)
    gen = torch.Generator().manual_seed(6)
    dr, dh = (torch.randn(r.shape, generator=gen).bfloat16() for _ in range(2))
    entry.backward(mu, *s.backward(mu, dr.cuda(), dh.cuda()))
    wr, wh, leaf, norms = plain(s, entry, tokens, mu)
    assert off(r, wr) < 0.02 and off(hr, wh) < 0.02
    torch.autograd.backward([wr, wh], [dr.double(), dh.double()])
    got = dict(s.gradients, table=torch.cat(entry.gradients), pre=entry.pre_gradient, wq=s.head_gradients[0], wk=s.head_gradients[1])
    for k, w in leaf.items():
        assert off(got[k], w.grad) < 0.05, k
    for n, g in zip(norms, s.norm_gradients):
        for k in n:
            assert off(g[k], n[k].grad) < 0.05, k
    assert not s.kept and not entry.kept


def test_the_order_of_a_schedule_changes_nothing(stage):
    """nor does it draw other masks"""
    sizes, more = (3, 6, LENGTHS, 128, 4, 2, 256, True), {"turning": TURNING, "rate": RATE}
    _, _, operations = stage.plan(3, (1.0, 2.1), 3, 9, 6, max_nr=3)
    result = []
    for ops in (operations, stage.in_turn(3, 6)):
        stages, packings, xs, _ = stage.make(*sizes, **more)
        entry, tokens = stage.make_entry(6, LENGTHS, 128, 1000, 3, rate=RATE)
        dr = torch.ones_like(xs[0])
        back = stage.run(stages, packings, None, None, lambda mu, r, h: (dr, h), ops, entry, tokens)
        result.append([t for pair in back for t in pair] + entry.gradients + [entry.pre_gradient] + [t for s in stages for t in (*s.gradients.values(), *s.head_gradients)])
    # (gradients are sums over micro-batches, whose backward passes are in the same order in both)
    assert all(torch.equal(a, b) for a, b in zip(*result))


def test_shards_are_the_whole(stage):
    """one table or five shards of it: the same stream, the same gradients, bit by bit"""
    whole, (tokens,) = stage.make_entry(1, [700], 64, 333, 1, rate=RATE)
    parts, _ = stage.make_entry(1, [700], 64, 333, 5, rate=RATE)
    begin = 0
    for t in parts.tables:
        t.copy_(whole.tables[0][begin:begin + t.shape[0]])
        begin += t.shape[0]
    assert begin == 333
    d = torch.randn(700, 64, device="cuda").bfloat16()
    for a, b in zip(whole.forward(1, tokens), parts.forward(1, tokens)):
        assert torch.equal(a, b)
    for entry in (whole, parts):
        entry.backward(1, d, d)
    assert torch.equal(whole.gradients[0], torch.cat(parts.gradients)) and torch.equal(whole.pre_gradient, parts.pre_gradient)


def test_positions_of_a_packing(stage):
    from paper_2311_15269_amd import block_ops
    p = block_ops.Packing([3, 0, 1, 4], total_tokens=10)
    assert p.positions.tolist() == [0, 1, 2, 0, 0, 1, 2, 3, 0, 0] and p.positions is p.positions
    assert block_ops.Packing([]).positions.shape == (0,)


def test_positions_of_a_packing_that_is_gone(stage):
    """made on one stream, read on another that is busy, and the packing dropped: the first stream's next tensors do not get their memory"""
    from paper_2311_15269_amd import block_ops
    n, gen = 5000, torch.Generator(device="cuda")
    gen.manual_seed(2)
    q, k = (torch.randn(n, h, 64, generator=gen, device="cuda").bfloat16() for h in (4, 2))
    f, (busy, product) = block_ops.frequencies(64), (torch.zeros(8192, 8192, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    want = block_ops.rotate(q, k, torch.arange(n, device="cuda"), f)
    torch.mm(busy, busy, out=product)
    torch.cuda.synchronize()
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(first):
        packing = block_ops.Packing([n])
        at = packing.positions.data_ptr()
    with torch.cuda.stream(second):
        for _ in range(100):
            torch.mm(busy, busy, out=product)
        got = block_ops.rotate(q, k, packing.positions, f)
    del packing
    with torch.cuda.stream(first):
        others = [torch.full((n,), 7, dtype=torch.int32, device="cuda") for _ in range(8)]
    if not second.query():                                      # (once it is done the memory is anyone's)
        assert at not in [t.data_ptr() for t in others]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_captured_step(stage):
    """lookup, dropout, norms, rotation, attention and back to the table's gradient in one graph, with other tokens and other masks in each replay"""
    from paper_2311_15269_amd import block_ops
    packing = block_ops.Packing(LENGTHS)
    n, gen = sum(LENGTHS), torch.Generator(device="cuda")
    gen.manual_seed(1)
    table = torch.randn(400, 4 * 64, generator=gen, device="cuda").bfloat16()
    tokens, step = torch.randint(0, 400, (n,), generator=gen, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    w, f, positions = torch.ones(64, device="cuda"), block_ops.frequencies(64), packing.positions
    d = torch.randn(n, 2, 64, generator=gen, device="cuda").bfloat16()
    drop = block_ops.Dropout(0.3, 9, 0, step)

    def training_step():
        x = block_ops.embed(tokens, table, 2.0, 0, drop).view(n, 4, 64)
        q, k = block_ops.rotate(x[:, :2], x[:, 2:3], positions, f, w, w)
        o, lse = packing.attention(q, k, x[:, 3:])
        dq, dk, dv = packing.attention_backward(d, q, k, x[:, 3:], o, lse)
        dx = torch.empty_like(x)
        _, _, dwq, dwk = block_ops.rotate_backward(dq, dk, x[:, :2], x[:, 2:3], positions, f, w, w, out=(dx[:, :2], dx[:, 2:3]))
        dx[:, 3:] = dv
        dtable = block_ops.embed_backward(dx.view(n, -1), tokens, 400, 2.0, 0, drop)
        return o, dwq, dwk, dtable
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        training_step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = training_step()
        step += 1
    step.zero_()
    seen = []
    for k in range(4):
        tokens.copy_(torch.randint(0, 400, (n,), generator=gen, device="cuda"))
        step.fill_(k)
        want = training_step()
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == k + 1
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        seen.append(got[0].clone())
    assert not any(torch.equal(seen[0], t) for t in seen[1:])
