"""Attention over a window at the sizes of whole prompt pieces and wide groups, and the precision of its weights."""
import numpy as np
import pytest
import torch

from oracle import kv8
from tests.test_gpu_window import _gen, _i32, _tree, _words, check, hide, history, keys_of, make, positions, queries, seen_by, step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page,d,H_kv,G,T,window,sinks", [
    (16, 128, 1, 4, 1024, 256, 4), (0, 64, 2, 2, 2048, 1000, 0), (64, 128, 2, 1, 600, 4096, 16), (5, 64, 1, 8, 512, 100, 3), (32, 64, 1, 1, 4096, 33, 1),
])
def test_long_pieces(bits, page, d, H_kv, G, T, window, sinks):
    """Hundreds to thousands of queries, before, at and behind the cache's first tokens; every 61st query compared."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(T + d)
    lens, room = [T + 700, T, T // 2 + 3], T + 704
    cache = make(ssb, bits, len(lens), H_kv, d, page, room, 5)
    Q = queries(g, len(lens), H_kv * G, T, d, "bthd")
    hide(cache, lens, T, window, sinks, room)
    O, LSE = step(ssb, bits, cache, Q, lens, window, sinks)
    some = set(range(0, T, 61)) | {0, 1, T - 1, T // 2 - 4, T // 2 - 3, T // 2 - 2}
    check(Q, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks), d ** -0.5, bits, lambda b, h, t: t in some)
    for b, n in enumerate(lens):                               # queries in front of the request's first token
        none = max(0, T - n)
        assert (O[b, :, :none] == 0).all() and (LSE[b, :, :none] == -float("inf")).all()
        assert torch.isfinite(O[b].float()).all() and torch.isfinite(LSE[b, :, none:]).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d,H_kv,G,T", [(128, 1, 32, 1), (64, 1, 128, 1), (128, 2, 16, 3), (64, 32, 1, 1), (128, 40, 1, 5), (64, 1, 71, 2)])
def test_wide_groups_and_many_heads(bits, d, H_kv, G, T):
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(G + T)
    lens, room = [650, 0, 17, 333], 672
    cache = make(ssb, bits, 4, H_kv, d, 16, room, 5)
    Q = queries(g, 4, H_kv * G, T, d)
    hide(cache, lens, T, 90, 4, room)
    O, LSE = step(ssb, bits, cache, Q, lens, 90, 4, kernel="tcgen05")
    check(Q, O, LSE, keys_of(cache, H_kv, lens, T, 90, 4), d ** -0.5, bits, lambda b, h, t: h % 7 == 0)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d,H_kv,G,T", [(128, 2, 4, 64), (64, 2, 2, 130)])
def test_wide_trees(bits, d, H_kv, G, T):
    """Rounds over a window with trees of more nodes than the local kernel of few keys takes."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(T)
    lens, room, window, sinks = [900, 40, 300], 912, 200, 8
    B = len(lens)
    cache = make(ssb, bits, B, H_kv, d, 16, room, 5)
    Q, K, V = queries(g, B, H_kv * G, T, d), queries(g, B, H_kv, T, d), queries(g, B, H_kv, T, d)
    depth, seen = _tree(g, B, T)
    hide(cache, lens, T, window, sinks, room, depth, False)
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, room)
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    ctx.ss_verify_begin(Q, d ** -0.5)
    (ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window)(cache, window, sinks, _i32(lens), _i32(depth))
    ctx.ss_verify_local(K, V, ssb.SS_MASK_TREE_BITS, _words(seen))
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (0, 0)
    kl, vl = K.double().cpu().numpy(), V.double().cpu().numpy()
    local = lambda b, h, t: (kl[b, h][seen[b, t]], vl[b, h][seen[b, t]])
    check(Q, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks, depth, False, local), d ** -0.5, bits, lambda b, h, t: t % 5 == 0)
    ctx.close()


@pytest.mark.parametrize("d,G,T,bits,weight", [
    (128, 4, 1, 16, 2.0 ** -16), (128, 8, 2, 16, 2.0 ** -16), (64, 4, 8, 16, 2.0 ** -16),   # two bf16 terms
    (128, 4, 8, 16, 2.0 ** -8), (128, 24, 1, 16, 2.0 ** -8),                                # one
])
@pytest.mark.parametrize("B,window", [(2, 700), (100, 200)])
def test_weights_are_as_precise_as_said(d, G, T, bits, weight, B, window):
    """A weight is off by `weight` of itself at most; besides, each relative to A = sum p |v|: the score's d products in
    fp32 (each partial sum off by 2^-23 of the sum of |q k|), its scaling and the reference's subtraction (2^-23 of the score,
    which is formed to base 2), the exponential (2^-22) and the sums of up to 1000 weights and of products in fp32 (2^-14).
    The output is rounded to bf16 (2^-8 of the value)."""
    from paper_2609_33184_b200 import binding as ssb
    g = _gen(d + G + T)
    H_kv, room = 1, 720
    lens = [720 - b % 31 for b in range(B)]
    cache = make(ssb, bits, B, H_kv, d, 16, room, 5)
    Q = queries(g, B, H_kv * G, T, d)
    scale = 0.25 * d ** -0.5                                   # scores near 0: all tokens weigh
    O, _ = step(ssb, bits, cache, Q, lens, window, 0, scale, kernel="tcgen05")
    q, got = Q.double().cpu().numpy(), O.double().cpu().numpy()
    for b in range(0, B, 7):
        for t in range(T):
            k, v = (x[0] for x in history(cache, b, seen_by(positions(lens[b], T)[t], lens[b], window, 0)))
            o, _, A = kv8.attention(q[b, :, t], k, v, scale)
            s = scale * (np.abs(q[b, :, t]) @ np.abs(k).T).max(1, keepdims=True)
            tol = 2.0 ** -8 * np.abs(o) + (weight + d * 2.0 ** -23 * s + 2.0 ** -22 * s + 2.0 ** -22 + 2.0 ** -14) * A
            assert (np.abs(got[b, :, t] - o) <= tol).all(), (b, t, float((np.abs(got[b, :, t] - o) / tol).max()))
