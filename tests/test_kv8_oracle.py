"""Host-only checks of the 8-bit cache: the oracle's format against torch's own e4m3 conversion and the
definition, and the entry points' refusals that need no device."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2609_33184_b200 import binding as ssb
from paper_2609_33184_b200 import build as ssbuild


def test_code_values_are_e4m3():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, kv8.VALUES, equal_nan=True)


def test_encode_rounds_to_nearest_even():
    """Rows whose scale is 1 (a 448 among them) against torch's conversion, ties included."""
    x = torch.cat([torch.linspace(-448, 448, 5001), torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, 432.0])])
    x = x.bfloat16()
    row = torch.cat([x, torch.tensor([448.0]).bfloat16()])
    codes, byte = kv8.encode_row(row.double().numpy())
    assert byte == 127
    want = row.float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8.VALUES[codes], want)


@pytest.mark.parametrize("top,e", [(0.0, -32), (448.0, 0), (450.0, 1), (224.0, -1), (1.0, -8), (0.875, -9), (2.0 ** -40, -32),
                                   (3.3e38, 80), (float("inf"), -32)])
def test_exponent(top, e):
    assert kv8.exponent([0.0, -top, float("nan")]) == e


def test_values_survive_a_second_encoding():
    r = np.random.RandomState(0)
    for _ in range(200):
        x = torch.tensor(r.randn(64) * 2.0 ** r.randint(-12, 12)).bfloat16().double().numpy()
        once = kv8.decode(*kv8.encode_row(x))
        again = kv8.decode(*kv8.encode_row(once))
        assert np.array_equal(once, again)
        e = kv8.exponent(x)
        assert (np.abs(once - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (e - 10))).all()
        assert np.array_equal(torch.tensor(once).bfloat16().double().numpy(), once)   # every value is a bf16 value


def test_null_arguments_are_refused():
    ssbuild.build()
    lib = ssb.load()
    t = ssb.ss_tensor(None, 0, 0, 0)
    c = ssb.ss_cache8()
    assert lib.ss_kv8_write(None, C.byref(c), t, t, 1, 1, None, None, None, None) == ssb.SS_ERR_ARG
    assert lib.ss_kv8_read(None, C.byref(c), t, t, 1, 1, None, None, None) == ssb.SS_ERR_ARG
    assert lib.ss_verify_chunk8(None, C.byref(c), None, None) == ssb.SS_ERR_ARG
    assert lib.ss_decode8(None, t, 1, 1, 1.0, C.byref(c), None, None, None, None) == ssb.SS_ERR_ARG
