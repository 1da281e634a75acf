"""The operators between the tokens and the attention from their definitions, in 64 bits on the CPU, with bounds on what rounding may do.

H is half a step of a 32-bit number as a share of its value.  A sum of n terms in 32 bits, in any order, is at most n H times the sum of the
terms' sizes off (to first order; every bound below leaves room for the second).
"""
from fractions import Fraction

import numpy as np
import torch

H = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def philox(counter, key):
    """Philox4x32-10 of four and two numbers"""
    c, k = [int(n) for n in counter], [int(n) for n in key]
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [q >> 32 ^ c[1] ^ k[0], q & 0xFFFFFFFF, p >> 32 ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def words(tokens, channels, seed, number):
    """the random words of [tokens, channels]"""
    return words_of(np.arange(tokens), channels, seed, number)


def words_of(places, channels, seed, number):
    """those of the tokens at these places"""
    n, groups = len(places), -(-channels // 4)
    x = np.zeros((4, n, groups), np.uint64)
    x[0] += np.arange(groups, dtype=np.uint64)
    x[1] += np.asarray(places, dtype=np.uint64)[:, None]
    x[2] += np.uint64(number % 2 ** 32)
    x[3] += np.uint64(number >> 32)
    k = [seed % 2 ** 32, seed >> 32]
    low, by = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = np.stack([q >> by ^ x[1] ^ np.uint64(k[0]), q & low, p >> by ^ x[3] ^ np.uint64(k[1]), p & low])
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.moveaxis(x, 0, -1).reshape(n, -1)[:, :channels]


def kept(tokens, channels, rate, seed, number):
    """(what is kept, the factor of 32 bits)"""
    rate = float(np.float32(rate))
    keep = words(tokens, channels, seed, number % 2 ** 64) >= np.uint64(int(rate * 2 ** 32))
    return torch.from_numpy(keep), torch.tensor(1 / (1 - rate), dtype=torch.float32)


def dropped(x, rate, seed, number):
    """dropout of x bit by bit: one product in 32 bits, rounded once"""
    keep, by = kept(*x.shape, rate, seed, number)
    return torch.where(keep, x.float() * by, torch.zeros(())).to(x.dtype)


def embedding(token, table, scale, first, drop=None):
    """what embed() gives, bit by bit: products in 32 bits, rounded once; drop: (rate, seed, number)"""
    out = torch.zeros(token.shape[0], table.shape[1])
    for t, n in enumerate(token.tolist()):
        if first <= n < first + table.shape[0]:
            out[t] = table[n - first].float() * torch.tensor(scale, dtype=torch.float32)
    if drop:
        keep, by = kept(*out.shape, *drop)
        out = torch.where(keep, out * by, torch.zeros(()))
    return out.to(table.dtype)


def embedding_gradient(d_out, token, rows, scale, first, drop=None):
    """the gradient in 64 bits and its bound: a term's factor and the scale round once each, n terms add up"""
    d = d_out.double()
    if drop:
        keep, by = kept(*d.shape, *drop)
        d = torch.where(keep, d * by.double(), torch.zeros((), dtype=torch.float64))
    out, size, n = torch.zeros(rows, d.shape[1], dtype=torch.float64), torch.zeros(rows, d.shape[1], dtype=torch.float64), torch.zeros(rows, 1)
    at = token.long() - first
    there = (at >= 0) & (at < rows)
    out.index_add_(0, at[there], d[there] * scale)
    size.index_add_(0, at[there], d[there].abs() * abs(scale))
    n.index_add_(0, at[there], torch.ones(int(there.sum()), 1))
    return out, (n + 3) * H * size + 2.0 ** -149


def pairs(dim, turning, neighbours):
    """the channels of the pairs that turn"""
    i = torch.arange(turning // 2)
    return (2 * i, 2 * i + 1) if neighbours else (i, i + turning // 2)


def turned(z, angle, dim, turning, neighbours):
    """z [tokens, heads, dim] with its pairs turned by angle [tokens, pairs]"""
    a, b = pairs(dim, turning, neighbours)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    out = z.clone()
    out[..., a] = z[..., a] * cos - z[..., b] * sin
    out[..., b] = z[..., a] * sin + z[..., b] * cos
    return out


def both(z, dim, turning, neighbours):
    """sizes of what a turned channel is made of"""
    a, b = pairs(dim, turning, neighbours)
    out = z.abs().clone()
    out[..., a] = out[..., b] = z[..., a].abs() + z[..., b].abs()
    return out


def rotation(z, position, frequency, w, eps, neighbours, d=None):
    """(out, dz, dw) of one of queries and keys, and their bounds.

    Sines and cosines: the angle in turns is off by two roundings of 64 bits (position frequency 2^-52), its fraction is rounded to 32 bits (2^-25 of half
    a turn, 2^-23 as an angle), and they are rounded themselves by a few steps (2^-23): 2^-21 with what the products add.  A root mean square: dim terms, a division and a
    root: (dim / 2 + 4) H.  The mean that is taken off going back: dim H of the sum of its terms' sizes, and the root's error three times."""
    t, (n, heads, dim) = z.dtype, z.shape
    turning = 2 * len(frequency)
    angle = position.double()[:, None] * frequency
    off = 2.0 ** -21 + 2.0 ** -50 * (angle.abs().amax() if angle.numel() else 0.0)
    x = z.double()
    over = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) if w is not None else torch.ones(n, heads, 1, dtype=torch.float64)
    xn = x * over
    e = (dim / 2 + 4) * H if w is not None else 0.0
    y = xn * w.double() if w is not None else x
    out = turned(y, angle, dim, turning, neighbours)
    size = both(y, dim, turning, neighbours)
    result = [(out, U[t] * out.abs() * (1 + 1e-3) + TINY[t] + (off + e + 6 * H) * size)]
    if d is None:
        return result
    g = turned(d.double(), -angle, dim, turning, neighbours)
    gs = both(d.double(), dim, turning, neighbours)
    if w is None:
        return result + [(g, U[t] * g.abs() * (1 + 1e-3) + TINY[t] + (off + 6 * H) * gs), (None, None)]
    dw, dws = (g * xn).sum((0, 1)), (gs * xn.abs()).sum((0, 1))
    a, s = g * w.double(), gs * w.double().abs()
    dz = over * (a - xn * (a * xn).mean(-1, keepdim=True))
    size = over * (s + xn.abs() * (s * xn.abs()).mean(-1, keepdim=True))
    return result + [(dz, U[t] * dz.abs() * (1 + 1e-3) + TINY[t] + (off + dim * H + 3 * e + 12 * H) * size), (dw, (n * heads * H + off + e + 8 * H) * dws + 2.0 ** -149)]


def close(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs() - bound
    assert bool((off <= 0).all()), (what, float(off.max()), "of", float(want.abs().max()))


def reduced_angles(position, frequency):
    """position x frequency less whole turns, rounded once to 64 bits, from whole numbers of any length: [tokens, pairs] for lists of whole numbers and of 64-bit ones"""
    bits = 300                                                  # pi = 16 atan(1 / 5) - 4 atan(1 / 239) (Machin 1706)
    pi, power = 0, [0, 0]
    for i, (by, n) in enumerate(((16, 5), (-4, 239))):
        power[i], k = (1 << bits) // n, 0
        while power[i]:
            pi += (-1) ** k * by * (power[i] // (2 * k + 1))
            power[i], k = power[i] // n ** 2, k + 1
    turn = Fraction(2 * pi, 1 << bits)
    out = []
    for n in position:
        angles = [n * Fraction(f) for f in frequency]
        out.append([float(a - turn * round(a / turn)) for a in angles])
    return torch.tensor(out, dtype=torch.float64)
