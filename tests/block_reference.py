"""The block operators from their definitions, in 64 bits on the CPU, with bounds on what rounding may do to each value.

The bounds are first-order and hold for every element.  u is half a unit in the last place of the type (2^-9 bf16, 2^-12 f16 as a share of
a power of two: 2^-8 and 2^-11 of the value at most), and W the share by which 32-bit sums and the exponential may be off.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -23}
# the least a value of the type can be rounded by: half its smallest step
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
W = 2e-4          # 32-bit products of 128 terms, scores up to about 30, the exponential: 128 x 2^-24 x 30 is 2.3e-4 at worst


def attention(q, k, v, lengths, scale, d_o=None):
    """o, lse (and dq, dk, dv) of tensors on the CPU, and their bounds for inputs' type q.dtype, as two dicts"""
    t = q.dtype
    u, tiny = U[t], TINY[t]
    n, heads, dim = q.shape
    shared = heads // k.shape[1]
    Q, K, V = q.double(), k.double(), v.double()
    out = {"o": torch.zeros(n, heads, dim, dtype=torch.float64), "lse": torch.full((heads, n), -math.inf, dtype=torch.float64)}
    bound = {"o": torch.zeros(n, heads, dim, dtype=torch.float64), "lse": torch.zeros(heads, n, dtype=torch.float64)}
    if d_o is not None:
        D = d_o.double()
        for name, like in (("dq", Q), ("dk", K), ("dv", V)):
            out[name], bound[name] = torch.zeros_like(like), torch.zeros_like(like)
    begin = 0
    for length in lengths:
        at = slice(begin, begin + length)
        begin += length
        if length == 0:
            continue
        mask = torch.ones(length, length, dtype=torch.bool).tril()
        for h in range(heads):
            kv = h // shared
            s = (Q[at, h] @ K[at, kv].T * scale).masked_fill(~mask, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None]).masked_fill(~mask, 0.0)
            # products of queries and keys in 32 bits: what a probability may be off by
            w = W + (2.0 ** -22) * dim * scale * (Q[at, h].abs() @ K[at, kv].abs().T)
            out["o"][at, h], out["lse"][h, at] = p @ V[at, kv], lse
            # rounded probabilities (f16: those below its range against the row's largest, by a fixed amount), rounded result
            eo = (p * (u + 2 * w)) @ V[at, kv].abs() + length * tiny * 2 * V[at, kv].abs().amax(0) + u * (p @ V[at, kv]).abs() + tiny
            bound["o"][at, h], bound["lse"][h, at] = eo, w.amax(1) + 1e-6 * lse.abs() + 1e-6
            if d_o is None:
                continue
            g = D[at, h]
            dp = g @ V[at, kv].T
            delta = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - delta)
            out["dq"][at, h] += scale * ds @ K[at, kv]
            out["dk"][at, kv] += scale * ds.T @ Q[at, h]
            out["dv"][at, kv] += p.T @ g
            wide = dim * 2.0 ** -23 * (g.abs() @ V[at, kv].abs().T)
            off = (u + 2 * w) * ds.abs() + p * (wide + (p * (wide + 2 * w * dp.abs())).sum(1, keepdim=True) + (g.abs() * eo).sum(1, keepdim=True))
            off = off + (8 * tiny * (1 + d_o.double().abs().max()) if t == torch.float16 else 0.0) * mask
            bound["dq"][at, h] += scale * off @ K[at, kv].abs()
            bound["dk"][at, kv] += scale * off.T @ Q[at, h].abs()
            bound["dv"][at, kv] += (p * (u + 2 * w) + (tiny if t == torch.float16 else 0.0) * mask).T @ g.abs()
    if d_o is not None:
        for name in ("dq", "dk", "dv"):
            bound[name] += (u + 1e-5) * out[name].abs() + tiny + 1e-6 * bound[name]
    return out, bound


def norm(x, y, pre, post, gate, scale, eps, dr=None, dh=None):
    """dict of the outputs of the residual norm and of its backward pass, by torch's differentiation in 64 bits"""
    v = {name: t.detach().double().clone().requires_grad_(dr is not None) for name, t in (("x", x), ("y", y), ("pre", pre), ("post", post), ("gate", gate)) if t is not None}

    def n(z, w):
        return w * z / torch.sqrt((z * z).mean(1, keepdim=True) + eps)
    u = n(v["y"], v["post"]) if post is not None else v["y"]
    r = scale * v["x"] + (u * v["gate"] if gate is not None else u)
    h = n(r, v["pre"])
    out = {"r": r.detach(), "h": h.detach()}
    if dr is not None:
        got = torch.autograd.grad([r, h], list(v.values()), [dr.double(), dh.double()])
        out.update(("d" + name, g) for name, g in zip(v, got))
    return out


def held(x):
    """(whole numbers, exponents) of a checkpoint of x, group by group, -1000 for a group that is not finite"""
    least = -24 if x.dtype == torch.float16 else -126
    top = torch.finfo(x.dtype).max
    n, c = x.shape
    groups = -(-c // 64)
    whole = torch.zeros(n, c, dtype=torch.float64)
    exponent = torch.zeros(n, groups, dtype=torch.int64)
    for g in range(groups):
        part = x[:, 64 * g:64 * g + 64].double()
        for i in range(n):
            most = float(part[i].abs().max())
            if not math.isfinite(most):
                exponent[i, g] = -1000
                continue
            e = least
            while not most < 127.5 * 2.0 ** e:
                e += 1
            exponent[i, g] = e
            q = torch.round(part[i] / 2.0 ** e)
            limit = int(top / 2.0 ** e) if top / 2.0 ** e < 127 else 127
            whole[i, 64 * g:64 * g + 64] = q.clamp(-limit, limit)
    return whole, exponent


def values(whole, exponent):
    step = torch.where(exponent == -1000, torch.tensor(math.nan, dtype=torch.float64), torch.exp2(exponent.double()))
    return whole * step.repeat_interleave(64, 1)[:, :whole.shape[1]]


def act(kind, z):
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))) / 2
