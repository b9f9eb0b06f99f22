"""Depths of a round's candidates over a window: the query of depth 0 may be any; a request without one is reported."""
import pytest
import torch

from tests.test_gpu_window import _gen, _i32, check, hide, keys_of, make, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _round(ssb, bits, cache, Q, lens, window, sinks, depth):
    B, H_q, T, d = Q.shape
    ctx = ssb.Context(B, H_q, cache.H_kv, d, T, T, cache.desc.page_size * cache.desc.pages_per_req)
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    ctx.ss_verify_begin(Q, d ** -0.5)
    (ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window)(cache, window, sinks, _i32(lens), _i32(depth))
    ctx.ss_verify_finalize(O, LSE)
    status = ctx.ss_poll_status()
    ctx.close()
    return O, LSE, status


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [16, 5])                      # tensor cores, CUDA cores
@pytest.mark.parametrize("B,lens,T,G,d,window", [(3, (700, 130, 9), 5, 4, 128, 40), (2, (700, 33), 40, 2, 64, 9), (170, None, 3, 2, 64, 60)])
def test_any_query_may_have_depth_0(bits, page, B, lens, T, G, d, window):
    """Depths in any order; what no query sees is NaN, pages without a seen token have wrong ids."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(T + page)
    lens = list(lens) if lens else [int(x) for x in torch.randint(0, 700, (B,), generator=g)]
    depth = []
    for b in range(B):
        row = [0] + [int(x) for x in torch.randint(0, T, (T - 1,), generator=g)]
        depth.append([row[i] for i in torch.randperm(T, generator=g).tolist()])
    assert any(row[0] for row in depth)
    cache = make(ssb, bits, B, 2, d, page, 720, 5)
    Q = queries(g, B, 2 * G, T, d)
    hide(cache, lens, T, window, 2, 720, depth, False)
    O, LSE, status = _round(ssb, bits, cache, Q, lens, window, 2, depth)
    assert status == (0, 0)
    only = None if B < 10 else (lambda b, h, t: b % 17 == 0)
    check(Q, O, LSE, keys_of(cache, 2, lens, T, window, 2, depth, False), d ** -0.5, bits, only)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("B,T,d,tokens,window", [(1, 3, 128, 600, 50), (4, 70, 64, 600, 300), (200, 2, 64, 300, 100), (1, 4, 64, 9000, 8800)])
def test_a_request_without_depth_0_is_reported(bits, page, B, T, d, tokens, window):
    """Values as the formula says where all that is read is finite, and the flag, whatever form the call takes."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(B)
    cache = make(ssb, bits, B, 1, d, page, tokens, 5)
    lens = [tokens - b % 5 for b in range(B)]
    depth = [list(range(T)) for _ in range(B)]
    Q = queries(g, B, 2, T, d)
    assert _round(ssb, bits, cache, Q, lens, window, 2, depth)[2] == (0, 0)
    depth[B // 2] = [max(1, t) for t in range(T)]
    O, LSE, status = _round(ssb, bits, cache, Q, lens, window, 2, depth)
    assert status == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_DEPTH)
    check(Q, O, LSE, keys_of(cache, 1, lens, T, window, 2, depth, False), d ** -0.5, bits, lambda b, h, t: b == B // 2 and t % 9 == 0)
