"""Dropout and the embedding of batches so large that a lane takes four tokens -- in 16 bits with dropout from 2^22 chunks of eight channels on, a dropout by itself in rows of up to 256 channels, and
wherever rows take more lanes than a launch has -- whose numbers of tokens are no multiples of what a lane or a wave takes; and gradients of shards whose rows go on over many runs, with
factors that 32 bits round."""
import numpy as np
import pytest
import torch

from tests import entry_reference as R

pytestmark = pytest.mark.gpu
# rows of whole waves, a last tile that is full, nearly empty and of one channel; rows of fewer lanes, of one and of two counters, of fewer than eight channels
SIZES = [(8177, 4104), (8178, 4097), (8195, 4096), (65539, 512), (127103, 257), (131075, 256), (838861 + 30, 40), (838861 + 33, 37), (2097152 + 63, 9), (4194304 + 101, 8), (4194304 + 255, 5),
         (4194304 + 1, 4), (4194304 + 130, 1)]


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2311_15269_amd import block_ops
    return block_ops


def some(n):
    """places of the first tokens, of a few in the middle and of the last ones"""
    return sorted(set(range(9)) | {n // 3, n // 2, n // 2 + 1} | set(range(n - 300, n)))


def dropped_at(places, x, rate, seed, number):
    """dropout bit by bit of the rows x, which stand at these places"""
    rate = float(np.float32(rate))
    keep = torch.from_numpy(R.words_of(places, x.shape[1], seed, number) >= np.uint64(int(rate * 2 ** 32)))
    return torch.where(keep, x * torch.tensor(1 / (1 - rate), dtype=torch.float32), torch.zeros(()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n, c", SIZES)
def test_dropout(ops, n, c, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n)
    room = torch.full((n + 1, c), 7.0, dtype=dtype, device="cuda")
    x, drop, at = room[:n].copy_(torch.randn(n, c, generator=gen, device="cuda")), ops.Dropout(0.3, 12345678901234567, (1 << 32) - 2), some(n)
    got = ops.dropout(x, drop)
    assert torch.equal(got, ops.dropout(x.float(), drop).to(dtype))                      # (32 bits: a token a lane, one product, rounded once)
    assert torch.equal(got[at].cpu(), dropped_at(at, x[at].cpu().float(), 0.3, 12345678901234567, (1 << 32) - 2).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n, c", SIZES)
def test_lookup(ops, n, c, dtype):
    """tokens of a shard, of others and of none, the last ones among them"""
    gen = torch.Generator(device="cuda").manual_seed(n + 1)
    table = torch.randn(50, c, generator=gen, device="cuda").to(dtype)
    token = torch.randint(80, 170, (n,), generator=gen, device="cuda")
    token[-1], token[-2], token[-5], token[0] = 149, -1, 100, 99
    drop, at = ops.Dropout(0.3, 99, 1 << 40), some(n)
    got = ops.embed(token, table, 1.7, 100, drop)
    assert torch.equal(got, ops.embed(token, table.float(), 1.7, 100, drop).to(dtype))
    rows = token[at].cpu() - 100
    there = (rows >= 0) & (rows < 50)
    want = torch.where(there[:, None], table.cpu().float()[rows.clamp(0, 49)] * torch.tensor(1.7), torch.zeros(()))
    assert torch.equal(got[at].cpu(), dropped_at(at, want, 0.3, 99, 1 << 40).to(dtype))


# a workgroup more than a launch holds with a token a lane, and some tokens more
FARTHEST = [((1 << 26) + 1, 257), ((1 << 26) + 1030, 264), ((1 << 30) + 67, 17)]


@pytest.mark.parametrize("n, c", FARTHEST)
def test_dropout_of_more_lanes_than_a_launch_has(ops, n, c):
    """all values with nothing dropped; with dropout the first and the last rows, and what is kept of all"""
    gen = torch.Generator(device="cuda").manual_seed(c)
    x = torch.empty(n, c, dtype=torch.bfloat16, device="cuda").uniform_(1, 2, generator=gen)
    y = ops.dropout(x, ops.Dropout(0.0, 1))
    step = 1 << 24
    assert all(torch.equal(x[t:t + step], y[t:t + step]) for t in range(0, n, step))
    del y
    at, y = some(n), ops.dropout(x, ops.Dropout(0.3, 5, 6))
    assert torch.equal(y[at].cpu(), dropped_at(at, x[at].cpu().float(), 0.3, 5, 6).bfloat16())
    kept = [(int((y[t:t + step] != 0).sum()), y[t:t + step].numel()) for t in range(0, n, step)]
    # (each a sum of m draws of 0.7: more than eight deviations off once in 10^15)
    assert all(abs(k - 0.7 * m) < 8 * (0.21 * m) ** 0.5 for k, m in kept)


@pytest.mark.parametrize("n, c", FARTHEST)
def test_lookup_of_more_lanes_than_a_launch_has(ops, n, c):
    table = torch.randn(7, c, generator=torch.Generator().manual_seed(c)).bfloat16()
    token = torch.randint(0, 9, (n,), dtype=torch.int32, device="cuda")
    out, step, g = ops.embed(token, table.cuda(), 0.5), 1 << 24, table.cuda()
    rows = torch.cat((g * 0.5, torch.zeros(2, c, dtype=torch.bfloat16, device="cuda")))
    assert all(torch.equal(out[t:t + step], rows[token[t:t + step]]) for t in range(0, n, step))


@pytest.mark.parametrize("n, c", [(700, 64), (3000, 1003), (20000, 40)])
def test_gradients_of_shards_and_of_the_whole(ops, n, c):
    """a third of the tokens one row, dropout by 1 / 0.7: shards and the whole table each within their bound of the sums in 64 bits, and the same bits twice"""
    gen = torch.Generator().manual_seed(n)
    token = torch.randint(-3, 340, (n,), generator=gen)
    token[torch.rand(n, generator=gen) < 0.33] = 201
    d = torch.randn(n, c, generator=gen).bfloat16()
    drop, g, at = ops.Dropout(0.3, 4, 5), d.cuda(), token.cuda()
    want, bound = R.embedding_gradient(d, token, 333, 0.37, 0, (0.3, 4, 5))
    parts = []
    for first in range(0, 333, 67):
        rows = min(67, 333 - first)
        once, again = (ops.embed_backward(g, at, rows, 0.37, first, drop) for _ in range(2))
        assert torch.equal(once, again)
        parts.append(once)
    R.close(torch.cat(parts), want, bound, "shards")
    R.close(ops.embed_backward(g, at, 333, 0.37, 0, drop), want, bound, "whole")
