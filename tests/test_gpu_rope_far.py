"""Angles at the ends of what a call accepts: frequencies up to 2^20 radians a position at any int32 position, against whole numbers.

A pair (1, 0) turns into (cos, sin) times the magnitude 1.  The reduced angle may be off by 2^-30 turns (5.9e-9 radians), the sine and cosine
of a right one by 5 u (u = 2^-24; see test_gpu_norm_rope.py), the products with 1 and 0 by none and the last sum by u.  The tests allow
7 u + 2^-30 turns."""
import math
from fractions import Fraction

import pytest
import torch

import test_gpu_norm_rope as rope_tests
from paper_2609_38984_b200 import swam

pytestmark = pytest.mark.gpu
BITS = 400


def pi_bits():
    """floor(pi * 2^BITS) by Machin's formula: pi = 16 atan(1/5) - 4 atan(1/239)."""
    guard = 64
    one = 1 << (BITS + guard)

    def atan_inverse(x):
        total, term, n = 0, one // x, 1
        while term:
            total += term // n if n % 4 == 1 else -(term // n)
            term //= x * x
            n += 2
        return total

    return (16 * atan_inverse(5) - 4 * atan_inverse(239)) >> guard


def reduced(freq, position, pi):
    """freq * position modulo 2 pi in [-pi, pi], as a float."""
    two_pi = Fraction(2 * pi, 1 << BITS)
    angle = Fraction(freq) * position
    return float(angle - round(angle / two_pi) * two_pi)


def test_the_whole_range_of_frequencies_and_positions():
    pi = pi_bits()
    assert abs(pi / (1 << BITS) - math.pi) < 1e-15
    D = 32
    freq = [2.0 ** 20, -2.0 ** 20, 1048575.3, 777777.7, 123456.789, 1e5, 31415.9, 1000.5, 801.25, 100.1, 10.7, 1.0, 0.1, 1e-3, 1e-6, 2.0 ** -31]
    assert len(freq) == D // 2
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -1999999999, 1 << 20, 131071, -77, 1, 0]
    x = torch.zeros(1, len(pos), 1, D, device="cuda")
    x[..., :D // 2] = 1
    ctx = rope_tests.ctx_for(1, 1, 1, D, torch.float32)
    got, _ = ctx.norm_rope(x, rope=swam.Rope(freq), positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    ctx.check()
    angle = torch.tensor([[reduced(f, p, pi) for f in freq] for p in pos], dtype=torch.float64)
    want = torch.cat([angle.cos(), angle.sin()], dim=1)
    err = (got[0, :, 0].double().cpu() - want).abs()
    tol = 7 * 2.0 ** -24 + 2 * math.pi * 2.0 ** -30
    assert (err <= tol).all(), [(pos[i], freq[j % 16], float(err[i, j])) for i, j in (err > tol).nonzero().tolist()[:8]]


@pytest.mark.parametrize("dtype", rope_tests.TYPES)
def test_rows_whose_squares_outgrow_32_bits_give_zeros(dtype):
    D = 64
    ctx = rope_tests.ctx_for(1, 2, 2, D, dtype)
    x = torch.randn(1, 3, 2, D, device="cuda")
    want, _ = ctx.norm_rope(x.to(dtype), rope=swam.Rope(rope_tests.ladder(D)), q_weight=torch.ones(D, device="cuda"))
    x[0, 1, 1] = 1e30
    got, _ = ctx.norm_rope(x.to(dtype), rope=swam.Rope(rope_tests.ladder(D)), q_weight=torch.ones(D, device="cuda"))
    assert (got[0, 1, 1] == 0).all()
    assert torch.equal(got[0, [0, 2]], want[0, [0, 2]]) and torch.equal(got[0, 1, 0], want[0, 1, 0])
