"""Host-only checks of the 8-bit cache's description."""
import torch

from oracle import kv8
from paper_2609_33184_b200 import binding as ssb


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
