"""Rotary positions far from 0, against turns in exact arithmetic: any frequency, positions up to 2^53.

Tolerance, before any run: the kernel's turn is position times frequency / 2 pi less its whole turns, to 2^-50 (two numbers in 64 bits hold
the product and 1 / 2 pi), which is nothing beside the rest: that of test_gpu_rotary at near positions, 2^-21 of |x1| + |x2|, and half a
step of the storage type."""
from fractions import Fraction

import pytest
import torch

from paper_2210_10246_amd import binding as B

pytestmark = pytest.mark.gpu


def pi(bits):
    """floor(pi 2^bits), by 16 atan(1/5) - 4 atan(1/239) (Machin) with 64 bits to spare."""
    one = 1 << bits + 64

    def atan_of_1_over(n):
        total = power = one // n
        k = 1
        while power:
            power //= -n * n
            k += 2
            total += power // k
        return total
    return 16 * atan_of_1_over(5) - 4 * atan_of_1_over(239) >> 64


def turns(position, frequency):
    """position frequency / 2 pi in (-1, 1), whole turns taken off: to float64's last bit."""
    bits = 400
    t = Fraction(position) * Fraction(frequency) * Fraction(1 << bits, 2 * pi(bits))
    return float(t - round(t))


def test_turns():
    assert pi(60) == int(3.141592653589793238463 * 2 ** 51) * 2 ** 9 + pi(60) % 2 ** 9      # float64's bits and what follows
    assert turns(0, 0.3) == 0.0 and abs(turns(1, 1.0) - 0.15915494309189535) < 1e-16
    assert abs(turns(355, 2.0) - 9.595e-6) < 1e-9 and turns(-355, 2.0) == -turns(355, 2.0)  # 355 / 113 is close to pi


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("first", [0, 2 ** 20 + 1, 2 ** 31 - 3, 2 ** 40 + 12345, 2 ** 48 - 1, 2 ** 53 - 4, -2 ** 53 + 2])
def test_far_positions_of_any_frequency(first, layout, dtype):
    S, half, heads = 3, 16, 2
    freqs = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    q = torch.randn(1, S, heads, 2 * half, generator=g, device="cuda").to(dtype)
    positions = first + torch.arange(S, device="cuda")[None]
    y, back = torch.empty_like(q), torch.empty_like(q)
    B.tempo_rotary_fwd(q, None, freqs.cuda(), positions, y, None, layout)
    B.tempo_rotary_bwd(q, None, freqs.cuda(), None, back, None, layout, 1.0, first)
    angle = 2 * torch.pi * torch.tensor([[turns(first + s, f) for f in freqs.tolist()] for s in range(S)], dtype=torch.float64,
                                        device="cuda")[None, :, None]
    c, n = angle.cos(), angle.sin()
    pairs = ((slice(0, half), slice(half, None)) if layout == "half" else (slice(0, None, 2), slice(1, None, 2)))
    x1, x2 = (q[..., p].double() for p in pairs)
    off = (x1.abs() + x2.abs()) * 2.0 ** -21
    for got, sign in ((y, 1), (back, -1)):
        for p, want in zip(pairs, (x1 * c - sign * x2 * n, x2 * c + sign * x1 * n)):
            over = (got[..., p].double() - want).abs() - off - want.abs() * torch.finfo(dtype).eps / 2
            assert bool((over <= 0).all()), float(over.max())
