"""Rotary positions as far as they go: the angle is that of the exact product of position and frequency."""
from fractions import Fraction

import numpy as np
import pytest

from test_step_operators import check, hl, ints, to_bits, to_f64, torch, up, values  # noqa: F401

TWO_PI = 2 * Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)


def turn(position, frequency):
    """What the angle leaves behind its whole turns, as a part of one, exactly and then rounded to 64 bits."""
    turns = Fraction(int(position)) * Fraction(float(frequency)) / TWO_PI
    return float(turns - round(turns))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,neighbours", [(64, False), (64, True), (36, False), (36, True)])
def test_the_angle_is_that_of_the_exact_product(hl, torch, dim, neighbours, dtype):  # noqa: F811
    """Frequencies up to 10^6 radians a position and positions at both ends of 32 bits.  fp32 sines and cosines of half turns: 4e-7 of |a| + |b|
    as for near positions."""
    rng = np.random.default_rng(41)
    tokens, pairs = 40, dim // 2
    pos = rng.integers(-2 ** 31, 2 ** 31, tokens).astype(np.int32)
    pos[:4] = 2 ** 31 - 1, -2 ** 31, 0, 2 ** 30 + 1
    freq = np.geomspace(1e6, 1e-4, pairs).astype(np.float32)
    bits = to_bits(rng.standard_normal((tokens, dim)), dtype)
    dev = up(torch, bits, dtype)
    out = torch.empty_like(dev)
    hl.apply_rotary(hl.Rotary(hl.BF16 if dtype == "bf16" else hl.FP16, tokens, dim, ints(torch, pos[None]), torch.from_numpy(freq).cuda(), dev, 1, out,
                              pairing=hl.PAIR_NEIGHBOURS if neighbours else hl.PAIR_HALVES))
    angle = 2 * np.pi * np.array([[turn(p, f) for f in freq] for p in pos])
    x = to_f64(bits.reshape(-1), dtype).reshape(tokens, dim)
    a, b = (x[:, 0::2], x[:, 1::2]) if neighbours else (x[:, :pairs], x[:, pairs:])
    got = values(out).reshape(tokens, dim)
    ga, gb = (got[:, 0::2], got[:, 1::2]) if neighbours else (got[:, :pairs], got[:, pairs:])
    tol = 4e-7 * (np.abs(a) + np.abs(b))
    check(ga, a * np.cos(angle) - b * np.sin(angle), tol, dtype)
    check(gb, b * np.cos(angle) + a * np.sin(angle), tol, dtype)
