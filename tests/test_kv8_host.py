"""Host-only checks of the 8-bit cache's description."""
import ctypes as C

import pytest
import torch

from oracle import kv8
from paper_2609_33184_b200 import binding as ssb
from paper_2609_33184_b200 import build as ssbuild


def test_an_empty_cache_holds_rows_of_zeros_in_the_format():
    K, V, Ks, Vs, table = ssb.Cache8.empty(3, 2, 16, 64, device="cpu").tensors
    codes, byte = kv8.encode_row([0.0] * 64)
    assert table is None and K.shape == V.shape == (3, 2, 16, 64) and Ks.shape == Vs.shape == (3, 2, 16)
    for t in (K, V):
        assert (t == torch.from_numpy(codes)).all()
    for t in (Ks, Vs):
        assert (t == byte).all()


def test_scale_bytes_outside_the_format_count_as_its_ends():
    for byte, e in ((0, -32), (94, -32), (95, -32), (127, 0), (207, 80), (208, 80), (255, 80)):
        assert kv8.decode([0x38], byte)[0] == 2.0 ** e   # code 1.0


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.int8, torch.bool])
def test_codes_of_another_type_are_refused(dtype):
    """Buffers of one byte per element that do not hold e4m3 codes."""
    good = ssb.Cache8.empty(2, 1, 8, 64, device="cpu").tensors
    for bad in (0, 1):
        t = list(good[:4])
        t[bad] = t[bad].to(torch.bool) if dtype is torch.bool else t[bad].view(dtype)
        with pytest.raises(AssertionError):
            ssb.Cache8(*t)
    ssb.Cache8(good[0].view(torch.float8_e4m3fn), good[1], good[2], good[3])


def _workspace(d, R, sets):
    cfg = ssb.ss_config(max_B=2, H_q=2 * R, H_kv=2, d=d, max_Tq=1, max_Tloc=1, max_Lc=256, max_chunks=sets, device=0, flags=0)
    return ssb.load().ss_workspace_bytes(C.byref(cfg))


@pytest.mark.parametrize("d,ctas", [(64, 444), (128, 296)])
def test_workspace_holds_the_states_of_the_ctas_that_can_run(d, ctas):
    """8 rows more per kv-head cost 8 rows in every partial set and two 8-bit states of 8 rows (m, l, room, a[d]) for
    each CTA of the largest attention launch: three CTAs per SM at head dim 64 with few rows, else two."""
    ssbuild.build()
    grow = {sets: _workspace(d, 16, sets) - _workspace(d, 8, sets) for sets in (4, 8)}
    per_set = (grow[8] - grow[4]) // 4
    scratch = grow[4] - 5 * per_set               # 4 sets and the local one
    assert abs(scratch - 2 * ctas * 8 * (d + 4) * 4) < 4096   # (areas are rounded up to 256 bytes)
