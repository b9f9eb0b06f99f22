"""Rotary positions without a GPU: the table of a rotation, its refusals, and the oracle."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import rope
from paper_2609_33184_b200 import binding as ssb
from paper_2609_33184_b200 import build as ssbuild

# pi to 90 digits
PI = Fraction("3.141592653589793238462643383279502884197169399375105820974944592307816406286208998628034825")


@pytest.fixture(scope="module", autouse=True)
def lib():
    ssbuild.build()
    return ssb.load()


@pytest.mark.parametrize("rot", [16, 48, 128])
def test_table_holds_revolutions(rot):
    """Units of 2^-64 revolutions, off by a unit and a half at most: half a unit of rounding, and 64 significant bits
    of numbers below one twice."""
    f = [1e6 ** (-2 * i / rot) for i in range(rot // 2)]
    f[:8] = [0.0, 1.0, -1.0, 2 * math.pi, 1e-30, -1e-30, 123456.789, -0.5]
    r = ssb.Rope(f, [i % 3 for i in range(rot // 2)], 3, True, 0.5).desc
    assert (r.rot_dim, r.n_axes, r.interleaved, r.magnitude) == (rot, 3, 1, 0.5)
    assert list(r.axis[: rot // 2]) == [i % 3 for i in range(rot // 2)]
    for i, x in enumerate(f):
        turns = Fraction(x) / (2 * PI)
        exact = (turns - math.floor(turns)) * 2 ** 64
        off = abs(exact - r.turn[i])
        off = min(off, 2 ** 64 - off)
        assert off <= Fraction(3, 2) * max(1, math.ceil(abs(turns))), (i, x, float(off))


@pytest.mark.parametrize("args,status", [
    ((8, 0, 1, [1.0] * 4, None, 1.0), ssb.SS_ERR_SHAPE),          # rot_dim no multiple of 16
    ((0, 0, 1, [1.0], None, 1.0), ssb.SS_ERR_SHAPE),
    ((144, 0, 1, [1.0] * 72, None, 1.0), ssb.SS_ERR_SHAPE),
    ((16, 0, 0, [1.0] * 8, None, 1.0), ssb.SS_ERR_SHAPE),
    ((16, 0, 5, [1.0] * 8, None, 1.0), ssb.SS_ERR_SHAPE),
    ((16, 0, 2, [1.0] * 8, [0] * 7 + [2], 1.0), ssb.SS_ERR_ARG),
    ((16, 0, 2, [1.0] * 8, [-1] + [0] * 7, 1.0), ssb.SS_ERR_ARG),
    ((16, 0, 1, [1.0] * 7 + [math.inf], None, 1.0), ssb.SS_ERR_ARG),
    ((16, 0, 1, [math.nan] + [1.0] * 7, None, 1.0), ssb.SS_ERR_ARG),
    ((16, 0, 1, [1.0] * 8, None, math.nan), ssb.SS_ERR_ARG),
    ((16, 0, 1, None, None, 1.0), ssb.SS_ERR_ARG),
])
def test_table_refusals(lib, args, status):
    rot, inter, axes, f, axis, m = args
    out = ssb.ss_rope()
    st = lib.ss_rope_init(C.byref(out), rot, inter, axes, None if f is None else (C.c_double * len(f))(*f),
                          None if axis is None else (C.c_int32 * len(axis))(*axis), m)
    assert st == status
    assert lib.ss_rope_init(None, 16, 0, 1, (C.c_double * 8)(*[1.0] * 8), None, 1.0) == ssb.SS_ERR_ARG


def test_calls_without_a_context_are_refused(lib):
    no = ssb.ss_tensor(None, 0, 0, 0)
    r = ssb.Rope([1.0] * 8)
    assert lib.ss_rope_rotate(None, r.ref, no, no, 1, 1, None, None, None, no, no, None) == ssb.SS_ERR_ARG
    assert lib.ss_kv_append(None, None, no, no, 1, 1, None, None, None, None, None, no, no, None) == ssb.SS_ERR_ARG
    assert lib.ss_kv8_append(None, None, no, no, 1, 1, None, None, None, None, None, no, no, None) == ssb.SS_ERR_ARG


def test_oracle_by_hand():
    x = np.array([[1.0, 2.0, 3.0, 4.0, 5.0]])
    f = [math.pi / 2, math.pi]
    half, size = rope.rotate(x, [[1, 1]], f)
    np.testing.assert_allclose(half, [[-3.0, -2.0, 1.0, -4.0, 5.0]], atol=1e-15)
    np.testing.assert_allclose(size, [[math.sqrt(10), math.sqrt(20), math.sqrt(10), math.sqrt(20), 0.0]])
    inter, _ = rope.rotate(x, [[1, 1]], f, True, 2.0)
    np.testing.assert_allclose(inter, [[-4.0, 2.0, -6.0, -8.0, 5.0]], atol=1e-14)
    back, _ = rope.rotate(rope.rotate(x, [[7, -9]], f)[0], [[-7, 9]], f)
    np.testing.assert_allclose(back, x, atol=1e-14)
    # scores depend on the difference of the positions alone
    q, k = np.array([[0.3, -1.0, 0.5, 2.0]]), np.array([[1.5, 0.2, -0.7, 0.4]])
    dot = lambda p: float((rope.rotate(q, [[p + 3] * 2], [1.0, 0.01])[0] * rope.rotate(k, [[p] * 2], [1.0, 0.01])[0]).sum())
    assert abs(dot(0) - dot(2 ** 31 - 9)) < 1e-8
