"""The 8-bit KV cache in fp64, from its definition (TEST INFRASTRUCTURE ONLY, see the package docstring).

A row is d codes in e4m3 (sign, 4 exponent bits with bias 7, 3 fraction bits, no infinities, 0x7f and
0xff are NaN) and one byte e + 127: a value is code * 2^e.  e is the smallest integer in [-32, 80] with
max|x| <= 448 * 2^e over the row's finite values; a byte outside [95, 207] counts as the nearer end.
"""
import numpy as np


def code_value(code: int) -> float:
    """Value of one e4m3 code."""
    sign, ex, fr = -1.0 if code & 0x80 else 1.0, (code >> 3) & 15, code & 7
    if ex == 15 and fr == 7:
        return float("nan")
    return sign * (fr * 2.0 ** -9 if ex == 0 else (8 + fr) * 2.0 ** (ex - 10))


VALUES = np.array([code_value(c) for c in range(256)])


def exponent(row) -> int:
    """e of one row (fp64 values)."""
    top = max((abs(float(x)) for x in row if np.isfinite(x)), default=0.0)
    e = -32
    while e < 80 and top > 448.0 * 2.0 ** e:
        e += 1
    return e


_POS = VALUES[:127]                                # codes 0x00 .. 0x7e in rising order


def encode_row(row):
    """-> (codes uint8 [d], byte): the nearest code, of two equally near ones the even one."""
    e = exponent(row)
    y = np.clip(np.asarray(row, dtype=np.float64) * 2.0 ** -e, -448.0, 448.0)
    mag = np.abs(y)
    hi = np.clip(np.searchsorted(_POS, np.nan_to_num(mag)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - mag, mag - _POS[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = np.where(mag == _POS[hi], hi, code).astype(np.uint8)
    code = np.where(np.isnan(y), 0x7F, code).astype(np.uint8)
    return code | np.where(np.signbit(y) & ~np.isnan(y), 0x80, 0).astype(np.uint8), e + 127


def decode(codes, byte):
    """codes [.., d], byte [..] -> fp64 values."""
    return VALUES[codes] * np.exp2(np.clip(np.asarray(byte, dtype=np.float64), 95.0, 207.0) - 127.0)[..., None]


def attention(q, K, V, scale):
    """q [R, d], K, V [n, d] fp64 -> O [R, d], LSE [R] and A = sum p |v| (what weight errors scale with)."""
    if K.shape[0] == 0:
        z = np.zeros((q.shape[0], V.shape[1]))
        return z, np.full(q.shape[0], -np.inf), z
    s = scale * (q @ K.T)
    m = s.max(axis=1, keepdims=True)
    p = np.exp(s - m)
    l = p.sum(axis=1, keepdims=True)
    return (p @ V) / l, (m + np.log(l))[:, 0], (p @ np.abs(V)) / l
