"""The table of a rotation at frequencies of many revolutions per position, and what it refuses."""
import math
import random
from fractions import Fraction

import pytest

from paper_2609_33184_b200 import binding as ssb
from paper_2609_33184_b200 import build as ssbuild

# pi to 90 digits
PI = Fraction("3.141592653589793238462643383279502884197169399375105820974944592307816406286208998628034825")


@pytest.fixture(scope="module", autouse=True)
def lib():
    ssbuild.build()
    return ssb.load()


def _off(f, units):
    """How far a table entry is from the frequency's revolutions, in units of 2^-64."""
    turns = Fraction(f) / (2 * PI)
    off = abs((turns - math.floor(turns)) * 2 ** 64 - units)
    return min(off, 2 ** 64 - off)


def test_table_is_the_nearest_unit_at_any_frequency():
    """Half a unit, and 2^-60 for pi's last digits (2^-298 of it) and the product's last place."""
    rng = random.Random(1)
    f = [0.0, 1.0, -1.0, 5e-324, 2.0 ** -62, 3.5e-19, -3.5e-19, 2 * math.pi, math.pi, -math.pi, 123456.789, 1e6, -1e6, 1e10, 1e15,
         2.0 ** 53, 1e18, -1e18, math.nextafter(2.0 ** 64, 0.0), -math.nextafter(2.0 ** 64, 0.0)]
    f += [rng.choice((-1, 1)) * math.exp(rng.uniform(-60.0, 44.0)) for _ in range(620)]
    for i in range(0, len(f), 64):
        part = f[i:i + 64]
        turn = ssb.Rope(part).desc.turn
        for x, t in zip(part, turn):
            assert _off(x, t) <= Fraction(1, 2) + Fraction(1, 2 ** 60), (x, t)


@pytest.mark.parametrize("f", [2.0 ** 64, -2.0 ** 64, 1e20, 1e300, math.inf, -math.inf, math.nan])
def test_frequencies_beyond_the_table_are_refused(f):
    with pytest.raises(ssb.SpecStreamError) as e:
        ssb.Rope([1.0] * 7 + [f])
    assert e.value.status == ssb.SS_ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("inter", [False, True])
def test_rotate_at_frequencies_of_many_revolutions(inter):
    """Frequencies up to 2^64 at far positions: one rounding to bf16 (2^-8 of the value) and 2^-20 of the pair's length."""
    import numpy as np
    import torch
    dev = "cuda:0"
    freq = [1e3, -4e4, 1e6, 123456.789, 1e9, 1e12, 1e15, 1.5e19]
    at = [1, -1, 131071, 2 ** 31 - 1, -2 ** 31, 1999999999]
    g = torch.Generator().manual_seed(3)
    x = torch.randn(1, 1, len(at), 64, generator=g).bfloat16()
    out = torch.empty_like(x, device=dev)
    ctx = ssb.Context(1, 1, 1, 64, 1, 1, 8)
    rope = ssb.Rope(freq, None, 1, inter)
    ctx.ss_rope_rotate(rope, x.to(dev), None, out, None, torch.tensor(at, dtype=torch.int32, device=dev).view(1, 1, -1))
    assert ctx.ss_poll_status() == (0, 0)
    ctx.close()
    x, got = x[0, 0].double().numpy(), out[0, 0].double().cpu().numpy()
    turn = [[float((Fraction(f) * p / (2 * PI)) % 1) * 2 * math.pi for f in freq] for p in at]
    c, s = np.cos(turn), np.sin(turn)
    one = 2 * np.arange(8) if inter else np.arange(8)
    two = one + 1 if inter else one + 8
    want, size = x.copy(), np.zeros_like(x)
    want[:, one], want[:, two] = x[:, one] * c - x[:, two] * s, x[:, one] * s + x[:, two] * c
    size[:, one] = size[:, two] = np.hypot(x[:, one], x[:, two])
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) * (size > 0) + 2.0 ** -20 * size).all()
