"""Attention over a window of a bf16 cache where a CTA goes through several units: every row holds its own unit's output."""
import pytest
import torch

from tests.test_gpu_window import _gen, _i32, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _signs(B, H_kv, d):
    """[B, H_kv, d]: the number of the (request, kv-head) pair in signs, once over every 16 head dims."""
    pair = torch.arange(B * H_kv).view(B, H_kv, 1)
    return 1.0 - 2.0 * (pair >> (torch.arange(d) % 16) & 1).double()


@pytest.mark.parametrize("form,B,H_kv,tokens,window", [
    ("window-tcgen05-whole", 260, 4, 120, 100), ("window-tcgen05-whole", 150, 8, 250, 200),   # units of one and two tiles
    ("window-tcgen05", 175, 2, 1536, 1500), ("window-tcgen05", 320, 1, 800, 700),             # units cut at shares' ends
])
@pytest.mark.parametrize("d,G,T", [(128, 8, 1), (128, 8, 4), (64, 4, 1), (64, 8, 4)])
@pytest.mark.parametrize("decode", [True, False])
def test_many_units_per_cta(form, B, H_kv, tokens, window, d, G, T, decode):
    """V is the same for all tokens of a unit, +1 or -1 by its number, so O is V: off by the weights' 2^-8 and the
    output's 2^-8 at most, where another unit's output is off by 2.  Outputs are cleared before each of many calls."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(B + d + T)
    want = _signs(B, H_kv, d).to(DEV)
    pages = -(-tokens // 32)
    table = torch.randperm(B * pages, generator=g).to(torch.int32).view(B, pages).to(DEV)
    cache = ssb.Cache16.empty(B * pages, H_kv, 32, d, table)
    K, V = cache.tensors[:2]
    K.normal_()
    for b in range(B):
        V[table[b].long()] = want[b, None, :, None, :].bfloat16()
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, pages * 32)
    Q, n = queries(g, B, H_kv * G, T, d), _i32([tokens - b % 9 for b in range(B)])
    rows = want.repeat_interleave(G, 1).unsqueeze(2).float()
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(300):
        O.fill_(9.0)
        LSE.fill_(float("nan"))
        if decode:
            ctx.ss_decode_window(Q, d ** -0.5, cache, window, 3, n, O, LSE)
        else:
            ctx.ss_verify_begin(Q, d ** -0.5)
            ctx.ss_verify_chunk_window(cache, window, 3, n)
            ctx.ss_verify_finalize(O, LSE)
        bad += ((O - rows).abs() > 2.0 ** -7).sum() + torch.isnan(LSE).sum()
    assert ctx.ss_poll_status() == (0, 0)
    assert int(bad) == 0
    assert ctx.last_chunk_kernel() == form
    ctx.close()
