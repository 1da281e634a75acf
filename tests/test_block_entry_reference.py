"""The reference of the operators between the tokens and the attention: random words by published ones, gradients by differences.  No GPU."""
import numpy as np
import pytest
import torch

from tests import entry_reference as R


def test_random_words():
    """published vectors of Philox4x32-10: all zeros, all ones"""
    assert R.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert R.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    seed, number = 0x123456789ABCDEF0, (5 << 32) + 0xFFFFFFFE
    w = R.words(7, 10, seed, number)
    for t, c in ((0, 0), (3, 5), (6, 9)):
        assert int(w[t, c]) == R.philox([c // 4, t, 0xFFFFFFFE, 5], [0x9ABCDEF0, 0x12345678])[c % 4]


def test_share_of_what_is_dropped():
    """of 2^18 values, as many as the rate says, by six standard deviations"""
    for rate in (0.1, 0.5, 0.9):
        keep, by = R.kept(512, 512, rate, 77, 3)
        n = keep.numel()
        assert abs(float(keep.float().mean()) - (1 - rate)) < 6 * (rate * (1 - rate) / n) ** 0.5
        assert float(by) == float(np.float32(1 / (1 - float(np.float32(rate)))))
    assert bool(R.kept(64, 64, 0.0, 1, 1)[0].all())


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_gradients_of_the_rotation_by_differences(neighbours, normed):
    gen = torch.Generator().manual_seed(3)
    z, d = (torch.randn(3, 2, 12, generator=gen, dtype=torch.float64) for _ in range(2))
    w = 1 + 0.3 * torch.randn(12, generator=gen, dtype=torch.float64) if normed else None
    f, position = torch.tensor([1.0, 0.3, 0.01, 2.0], dtype=torch.float64), torch.tensor([0, 5, 1000])
    R.U[torch.float64], R.TINY[torch.float64] = 0.0, 0.0

    def value(z, w):
        return float((R.rotation(z, position, f, w, 1e-3, neighbours)[0][0] * d).sum())
    _, (dz, _), (dw, _) = R.rotation(z, position, f, w, 1e-3, neighbours, d)
    h = 1e-6
    for i in (0, 5, 11, 30, 71):
        up, down = z.clone(), z.clone()
        up.view(-1)[i] += h
        down.view(-1)[i] -= h
        assert abs((value(up, w) - value(down, w)) / (2 * h) - float(dz.view(-1)[i])) < 1e-6
    for i in (0, 3, 11) if normed else ():
        up, down = w.clone(), w.clone()
        up[i] += h
        down[i] -= h
        assert abs((value(z, up) - value(z, down)) / (2 * h) - float(dw[i])) < 1e-6


def test_gradient_of_the_embedding_by_differences():
    gen = torch.Generator().manual_seed(4)
    table, d = torch.randn(5, 6, generator=gen), torch.randn(9, 6, generator=gen)
    token = torch.tensor([7, 3, 4, 4, -1, 8, 2, 4, 6])
    want, _ = R.embedding_gradient(d, token, 5, 0.5, 3, (0.25, 11, 12))

    def value(table):
        keep, by = R.kept(9, 6, 0.25, 11, 12)
        rows = torch.stack([0.5 * table[n - 3] if 3 <= n < 8 else torch.zeros(6, dtype=torch.float64) for n in token.tolist()])
        return float((rows * keep * float(by) * d.double()).sum())
    for i in range(30):
        up, down = table.double(), table.double()
        up.view(-1)[i] += 1e-3
        down.view(-1)[i] -= 1e-3
        assert abs((value(up) - value(down)) / 2e-3 - float(want.view(-1)[i])) < 1e-9


def test_angles_less_whole_turns():
    import math
    position, frequency = [0, 1, -1, 12, 1 << 30, 710], [1.0, 0.37, 1e-4]
    got = R.reduced_angles(position, frequency)
    want = torch.tensor([[math.remainder(n * f, 2 * math.pi) for f in frequency] for n in position], dtype=torch.float64)
    # (2 pi rounds by 2^-53 a turn, the product by 2^-53 of itself)
    assert float((got - want).abs().max()) < 2.0 ** -50 * (1 << 30) and float((got - want).abs()[[0, 1, 2, 3, 5]].max()) < 1e-12
    assert abs(math.sin(float(R.reduced_angles([1 << 62], [1.0])[0, 0])) - math.sin(1 << 62)) < 1e-15        # (the library's own reduction of a whole number of 64 bits)
