"""Calls of attention whose outputs show how the probabilities were rounded, and pins of what they show (no GPU).

Every key's score is one exact product. In each 16 rows one key has the largest score, 0, so that every part of a call
weighs its keys by the same p = exp(score); its value is 0. A value of another key is 1 or -1, as its p rounds up or down in bf16, and
some are left out so that the sums of both signs are nearly the same: the output is nearly 0, its own rounding nearly nothing, and
the roundings of the probabilities all add up.
"""

import numpy as np
import pytest


def rounded(p, bits):
    """p at `bits` significant bits (8: bf16, 11: fp16 where it is normal)."""
    _, e = np.frexp(p)
    return np.ldexp(np.rint(np.ldexp(p, bits - e)), e - bits)


def crafted(rng, n, scale, e4m3=False):
    """(keys' first element, signs of the values) of n rows (a multiple of 16), scores scale times the first."""
    if e4m3:
        least = np.concatenate([np.arange(8, 16) * 2.0 ** s for s in range(-5, 2)])      # e4m3 numbers 1/4 .. 30
        x = rng.choice(least, n) * (8 if scale >= 1 / 8 else 16) / 8
    else:
        x = rounded(rng.uniform(0.02, 3.0, n) / scale, 8)
    x[5::16] = 0
    p = np.exp(-scale * x)
    up = rounded(p, 8) - p
    sign = np.sign(up)
    sign[5::16] = 0
    # From the side with more weight only as much as the other has, the largest first.
    more = 1 if p[sign > 0].sum() > p[sign < 0].sum() else -1
    left = p[sign == -more].sum()
    for j in np.argsort(-p):
        if sign[j] == more:
            if p[j] <= left:
                left -= p[j]
            else:
                sign[j] = 0
    return -x, sign


def bound(ref, mass, n, prob, half):
    """What an output may be off by: half a step of its own, `prob` of what the probabilities weigh, 2^x and its argument (2^-19: three
    roundings of an argument below 8), and the fp32 sums of a product's steps of 16 keys, twice, and of 16 parts."""
    return half * np.abs(ref) + (prob * (1 + 2.0 ** -7) + 2.0 ** -19 + (n / 8 + 16) * 2.0 ** -23) * mass


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("scale", [1 / 8, 128.0 ** -0.5, 1 / 16])
def test_the_calls_tell_the_roundings_apart(e4m3, scale):
    n = 512
    for seed in range(5):
        x, v = crafted(np.random.default_rng(seed), n, scale, e4m3)
        p = np.exp(scale * x)
        ref, mass = (p * v).sum() / p.sum(), (p * np.abs(v)).sum() / p.sum()
        assert mass > 0.3 and abs(ref) < 0.01 * mass
        one = rounded(p, 8)
        off = [abs((y * v).sum() / p.sum() - ref) for y in (one, rounded(p, 11), one + rounded(p - one, 8))]
        most = [bound(ref, mass, n, prob, 2.0 ** -8) for prob in (2.0 ** -8, 2.0 ** -11, 2.0 ** -16)]
        assert off[0] <= most[0] and off[1] <= most[1] and off[2] <= most[2]
        assert off[0] > 1.5 * most[1] and off[0] > 8 * most[2]      # bf16 once shows where more bits are promised
