"""The 8-bit terms that the attention over the 8-bit cache multiplies with: how near their sums come to what they stand
for, by enumeration.  (The kernel forms them with the same roundings: e4m3 to nearest even with saturation, the upper
byte of an f16.)"""
import numpy as np
import torch


def e4m3(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.float8_e4m3fn).double().numpy()


def test_query_terms():
    """A query row is scaled by a power of two so that its maximum lies in (224, 448]; a value is hi + lo.  Every bf16 value
    down to 2^-30: exact from 1/4 on, that is 2^-9.8 of the smallest possible maximum (just above 224), and off by at most
    2^-10, that is 2^-17.8 of it, below."""
    bits = np.arange(1 << 15, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    x = x[(x >= 2.0 ** -30) & (x <= 448)].astype(np.float64)
    hi = e4m3(x)
    err = np.abs(hi + e4m3(x - hi) - x)
    assert (err[x >= 0.25] == 0).all()
    assert err[x < 0.25].max() <= 2.0 ** -10 and err[(x < 0.25) & (x > 0.24)].max() > 0
    assert 0.25 <= 2.0 ** -9.8 * 224 and 2.0 ** -10 <= 2.0 ** -17.75 * 224


def _byte(h):
    """e5m2 value of the upper byte of an f16."""
    return (h.view(np.uint16) & np.uint16(0xFF00)).view(np.float16)


def weight_terms(w):
    """fp32 weights -> hi + mid / 8 + lo / 64."""
    h = w.astype(np.float16)
    hi = _byte(h)
    a = ((h - hi) * np.float16(8)).astype(np.float16)
    mid = _byte(a)
    b = ((a - mid) * np.float16(8)).astype(np.float16)
    lo = _byte((b.view(np.uint16) + np.uint16(0x80)).view(np.float16))
    return hi.astype(np.float64) + mid.astype(np.float64) / 8 + lo.astype(np.float64) / 64


def test_weight_terms():
    """One part in 2^9 from the last term's rounding and one in 2^11 from that to f16, which above 2^-13 (2^-20 of a reference
    of 2^7) do not reach their largest at the same weight: 1.1 * 2^-9 together.  Below 2^-14 the error is at most 2^-23
    plus f16's 2^-25."""
    grain = np.arange(1 << 14, dtype=np.float64) / (1 << 14)
    for e in range(-14, 15):
        w = ((1 + grain) * 2.0 ** e).astype(np.float32)
        worst = (np.abs(weight_terms(w) - w) / w).max()
        assert 2.0 ** -9 < worst <= (1.25 if e == -14 else 1.1) * 2.0 ** -9, (e, worst * 2 ** 9)
    small = (np.arange(1 << 16) * 2.0 ** -30).astype(np.float32)
    assert np.abs(weight_terms(small) - small).max() <= 2.0 ** -23 + 2.0 ** -25
