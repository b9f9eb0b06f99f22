"""Attention over a window: refusals, device flags, values that are not finite, streams, capture, and whole steps."""
import numpy as np
import pytest
import torch

from oracle import kv8, rope
from tests import test_gpu_window as tw
from tests.test_gpu_window import _gen, _i32, check, history, keys_of, make, positions, queries, seen_by, step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ssb():
    from paper_2609_33184_b200 import binding
    return binding


def _put(cache, b, tokens, h, K=None, V=None):
    """fp64 rows for some tokens of a bf16 cache."""
    o, i = (torch.as_tensor(x, device=DEV) for x in tw.places(cache, b, tokens))
    for t, x in zip(cache.tensors, (K, V)):
        if x is not None:
            t[o, h, i] = torch.as_tensor(x, dtype=torch.float32).bfloat16().to(DEV)


# ------------------------------------------------------------------ references of the softmax

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d,G,T,window,sinks", [(64, 1, 200, 5, 0), (128, 2, 140, 3, 1), (64, 4, 1, 3000, 4), (128, 8, 1, 2900, 0), (128, 4, 8, 700, 200)])
@pytest.mark.parametrize("slope", [-0.5, 0.5, 3.0])
def test_scores_that_rise_fall_and_start_late(bits, d, G, T, window, sinks, slope):
    """Scores that change by `slope` a token (references are raised again and again, or all weight is in the first
    tokens), far from 0; rows that see nothing of their CTA's first tiles."""
    ssb = _ssb()
    B, H_kv, room = 2, 2, 3008
    lens = [3000, 517]
    g = _gen(d + T)
    cache = make(ssb, bits, B, H_kv, d, 32, room, 11)
    Q = torch.zeros(B, H_kv * G, T, d)
    Q[..., 0] = 1.0
    Q[..., 1:] = 0.05 * torch.randn(B, H_kv * G, T, d - 1, generator=g)
    Q = Q.bfloat16().to(DEV)
    K, V = torch.randn(B, H_kv, room, d, generator=g), torch.randn(B, H_kv, room, d, generator=g)
    K[..., 0] = slope * (torch.arange(room) - 1500.0)
    K, V = K.bfloat16().to(DEV), V.bfloat16().to(DEV)
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, 1, room)
    (ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append)(cache, K, V)
    O, LSE = step(ssb, bits, cache, Q, lens, window, sinks, 1.0, ctx)
    # (scores up to 4500: fp32 holds them to 2^-12, a weight to 2^-12 of itself)
    keys = keys_of(cache, H_kv, lens, T, window, sinks)
    q, Og, Lg = (x.double().cpu().numpy() for x in (Q, O, LSE))
    for b in range(B):
        for h in range(H_kv):
            for t in range(0, T, max(1, T // 9)):
                k, v = keys(b, h, t)
                for j in range(h * G, (h + 1) * G):
                    o, lse, A = kv8.attention(q[b, j, t][None], k, v, 1.0)
                    s = np.abs(q[b, j, t] @ k.T).max()
                    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -13 + s * 2.0 ** -20) * A + k.shape[0] * 2.0 ** -30 * np.abs(v).max()
                    assert (np.abs(Og[b, j, t] - o[0]) <= tol[0]).all(), (b, j, t)
                    low = 0.0
                    if bits == 8:
                        top = np.abs(q[b, j, t]).max()
                        low = (2.0 ** -17 * top * np.abs(k)).sum(1).max()
                    s_abs = (np.abs(q[b, j, t]) @ np.abs(k).T).max()
                    assert abs(Lg[b, j, t] - lse[0]) <= 2.0 ** -18 * s_abs + 2.0 ** -20 * abs(lse[0]) + 2.0 ** -16 + low, (b, j, t)
    ctx.close()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("kernel", ["tcgen05", "simt"])
@pytest.mark.parametrize("T", [1, 6])
@pytest.mark.parametrize("B,room", [(2, 1024), (160, 256)])
def test_values_that_are_not_finite(bits, kernel, T, B, room):
    """An infinite or NaN query makes its own row NaN; a NaN key those that see it; other rows keep their values."""
    ssb = _ssb()
    H_kv, G, d, page = 2, 4, 128, 16 if kernel == "tcgen05" else 5
    lens = [room - 24 - b % 7 for b in range(B)]
    window, sinks = 60, 2
    g = _gen(T)
    cache = make(ssb, bits, B, H_kv, d, page, room, 7)
    Q = queries(g, B, H_kv * G, T, d)
    clean, _ = step(ssb, bits, cache, Q, lens, window, sinks)
    Q2 = Q.clone()
    Q2[0, 1, T - 1, 5] = float("inf")
    Q2[0, 2, 0, 127] = -float("inf")
    Q2[1, 5, T - 1, 0] = float("nan")
    key = lens[1] - 20                                         # a key that all queries of request 1 see, on kv-head 0
    o, i = (int(x[0]) for x in tw.places(cache, 1, [key]))
    if bits == 8:
        cache.tensors[0][o, 0, i, 3] = 0x7F
    else:
        cache.tensors[0][o, 0, i, 3] = float("nan")
    O, LSE = step(ssb, bits, cache, Q2, lens, window, sinks, kernel=kernel)
    bad = torch.zeros(B, H_kv * G, T, dtype=torch.bool, device=DEV)
    bad[0, 1, T - 1] = bad[0, 2, 0] = bad[1, 5, T - 1] = True
    bad[1, :G] = True
    assert torch.isnan(O[bad]).all() and torch.isnan(LSE[bad]).all()
    assert not torch.isnan(O[~bad]).any() and not torch.isnan(LSE[~bad]).any()
    assert (O[~bad].float() - clean[~bad].float()).abs().max() <= 2.0 ** -6 * clean[~bad].float().abs().max()


# ------------------------------------------------------------------ device flags

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B,H_kv,window,page", [(4, 2, 90, 16), (4, 2, 90, 5), (200, 2, 90, 16), (1, 1, 9000, 16)])
def test_flags(bits, B, H_kv, window, page):
    """Lengths, pages and depths out of range are reported and clamped, read as zeros, clamped."""
    ssb = _ssb()
    d, G, T, sinks = 64, 2, 3, 4
    room = 9600 if B == 1 else 320
    g = _gen(B)
    cache = make(ssb, bits, B, H_kv, d, page, room, 3)
    table = cache.tensors[-1]
    room = cache.desc.page_size * cache.desc.pages_per_req
    lens = [room + 7 if b % 3 == 0 else -5 if b % 3 == 1 else 100 for b in range(B)]
    real = [min(max(n, 0), room) for n in lens]
    Q = queries(g, B, H_kv * G, T, d)
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, room)
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    decode = ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window
    decode(Q, 0.125, cache, window, sinks, _i32(lens), O, LSE)
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_VALID_LEN)
    only = None if B < 5 else (lambda b, h, t: b % 41 < 3)
    check(Q, O, LSE, keys_of(cache, H_kv, real, T, window, sinks), 0.125, bits, only)
    # page ids outside the pool: zeros
    last = (real[0] - 1) // page
    table[0, last] = cache.tensors[0].shape[0] if B < 100 else -1
    decode(Q, 0.125, cache, window, sinks, _i32(real), O, LSE)
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_PAGE)

    def keys(b, h, t):
        if h is None:
            return H_kv
        j = seen_by(positions(real[b], T)[t], real[b], window, sinks)
        gone = (b == 0) & (j // page == last)
        K, V = np.zeros((j.size, d)), np.zeros((j.size, d))
        if (~gone).any():
            k, v = history(cache, b, j[~gone])
            K[~gone], V[~gone] = k[h], v[h]
        return K, V
    check(Q, O, LSE, keys, 0.125, bits, (lambda b, h, t: b == 0) if B > 5 else None)
    # depths
    table[0, last] = 0
    depth = torch.tensor([[0, 7, -1]] * B, dtype=torch.int32)
    ctx.ss_verify_begin(Q, 0.125)
    (ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window)(cache, window, sinks, _i32(real), depth.to(DEV))
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_DEPTH)
    check(Q, O, LSE, keys_of(cache, H_kv, real, T, window, sinks, [[0, 2, 0]] * B, False), 0.125, bits, only)
    ctx.close()


def test_refusals():
    ssb = _ssb()
    B, H_kv, G, d, T = 2, 2, 2, 64, 2
    g = _gen(0)
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, 64)
    Q = queries(g, B, H_kv * G, T, d)
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    n = _i32([3, 40])
    c16, c8 = make(ssb, 16, B, H_kv, d, 16, 64, 0), make(ssb, 8, B, H_kv, d, 16, 64, 0)
    wide16, wide8 = make(ssb, 16, B, H_kv, d, 16, 80, 0), make(ssb, 8, B, H_kv, d, 0, 72, 0)

    def refused(status, f, *a):
        with pytest.raises(ssb.SpecStreamError) as e:
            f(*a)
        assert e.value.status == status

    for f, chunk, c, wide in ((ctx.ss_decode_window, ctx.ss_verify_chunk_window, c16, wide16),
                              (ctx.ss_decode8_window, ctx.ss_verify_chunk8_window, c8, wide8)):
        refused(ssb.SS_ERR_ARG, f, Q, 1.0, c, 0, 0, n, O, LSE)
        refused(ssb.SS_ERR_ARG, f, Q, 1.0, c, -3, 0, n, O, LSE)
        refused(ssb.SS_ERR_ARG, f, Q, 1.0, c, 5, -1, n, O, LSE)
        refused(ssb.SS_ERR_ARG, f, Q, 0.0, c, 5, 0, n, O, LSE)
        refused(ssb.SS_ERR_ARG, f, Q, float("inf"), c, 5, 0, n, O, LSE)
        refused(ssb.SS_ERR_SHAPE, f, Q, 1.0, wide, 5, 0, n, O, LSE)
        refused(ssb.SS_ERR_STATE, chunk, c, 5, 0)
        ctx.ss_verify_begin(Q, 1.0)
        refused(ssb.SS_ERR_STATE, f, Q, 1.0, c, 5, 0, n, O, LSE)
        refused(ssb.SS_ERR_ARG, chunk, c, 0, 0, n)
        refused(ssb.SS_ERR_SHAPE, chunk, wide, 5, 0, n)
        other = torch.cuda.Stream()
        refused(ssb.SS_ERR_STATE, chunk, c, 5, 0, n, None, other)
        with pytest.raises(AssertionError):
            chunk(c, 5, 0, n, _i32([0, 1]))                    # a depth for each query
        ctx.ss_verify_abort()
        for bad in (lambda: f(Q, 1.0, c, 5, 0, n.long(), O, LSE), lambda: f(Q, 1.0, c, 5, 0, n[:1], O, LSE),
                    lambda: f(Q.float(), 1.0, c, 5, 0, n, O, LSE), lambda: f(Q, 1.0, c, 5, 0, n, O[:, :, :1], LSE),
                    lambda: f(Q, 1.0, c, 5, 0, n, O, LSE.double()), lambda: f(Q, 1.0, c, 5, 0, n.cpu(), O, LSE),
                    lambda: f(Q, 1.0, c16 if c is c8 else c8, 5, 0, n, O, LSE), lambda: f(Q[:, :3], 1.0, c, 5, 0, n, O, LSE),
                    lambda: f(torch.cat([Q, Q]), 1.0, c, 5, 0, _i32([1] * 4), torch.cat([O, O]), torch.cat([LSE, LSE]))):
            with pytest.raises(AssertionError):
                bad()
        with pytest.raises(OverflowError):
            f(Q, 1.0, c, 2 ** 31, 0, n, O, LSE)
        f(Q, 1.0, c, 5, 0, None, O)                            # no lengths: all the room; no LSE
        assert ctx.ss_poll_status() == (0, 0)
    long = torch.zeros(B, H_kv * G, T + 1, d, dtype=torch.bfloat16, device=DEV)
    refused(ssb.SS_ERR_SHAPE, ctx.ss_decode_window, long, 1.0, c16, 5, 0, n, long.clone(), None)
    m, me = ctx._m, ctx._me
    with pytest.raises(TypeError):
        m.decode_window(me, Q)
    ctx.close()
    with pytest.raises(AssertionError):
        ctx.ss_decode_window(Q, 1.0, c16, 5, 0, n, O, LSE)


# ------------------------------------------------------------------ streams, capture, places

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B,window,room", [(3, 40, 512), (150, 60, 256), (1, 9000, 9600)])
def test_captured_steps_follow_the_lengths(bits, B, window, room):
    """A step and a round captured once on a stream of their own, replayed while the requests grow and shrink."""
    ssb = _ssb()
    H_kv, G, d, T = 2 if B > 1 else 1, 2, 64, 2
    g = _gen(B)
    cache = make(ssb, bits, B, H_kv, d, 16, room, 3)
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, room)
    Q, K_loc, V_loc = queries(g, B, H_kv * G, T, d), queries(g, B, H_kv, T, d), queries(g, B, H_kv, T, d)
    n = torch.zeros(B, dtype=torch.int32, device=DEV)
    out = [(torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)) for _ in range(4)]

    def run(a, b):
        (ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window)(Q, 0.125, cache, window, 3, n, *a)
        ctx.ss_verify_begin(Q, 0.125)
        (ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window)(cache, window, 3, n)
        ctx.ss_verify_local(K_loc, V_loc)
        ctx.ss_verify_finalize(*b)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run(*out[:2])
        for k in range(4):
            n.copy_(torch.randint(0, room + 1, (B,), generator=g, dtype=torch.int32) if k else torch.zeros(B, dtype=torch.int32))
            graph.replay()
            run(*out[2:])
            stream.synchronize()
            for x, y in zip(out[:2], out[2:]):
                assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
            lens = n.tolist()
            only = None if B < 5 else (lambda b, h, t: b % 50 == k)
            check(Q, *out[0], keys_of(cache, H_kv, lens, T, window, 3), 0.125, bits, only)
    assert ctx.ss_poll_status(stream) == (0, 0)
    ctx.close()


def test_two_contexts_side_by_side():
    """Two contexts on two streams at once give what each gives alone."""
    ssb = _ssb()
    d, H_kv, G, room = 128, 2, 4, 4096
    g = _gen(4)
    jobs = []
    for B, window, bits in ((2, 4000, 16), (60, 300, 8)):
        cache = make(ssb, bits, B, H_kv, d, 32, room if B < 10 else 512, B)
        Q = queries(g, B, H_kv * G, 1, d)
        n = _i32([int(x) for x in torch.randint(1, cache.desc.page_size * cache.desc.pages_per_req, (B,), generator=g)])
        ctx = ssb.Context(B, H_kv * G, H_kv, d, 1, 1, room)
        f = ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window
        jobs.append((f, Q, cache, window, n, torch.cuda.Stream(), ctx))
    out = []
    for f, Q, cache, window, n, s, ctx in jobs:
        O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
        f(Q, 0.1, cache, window, 4, n, O, LSE)
        out.append((O, LSE))
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for f, Q, cache, window, n, s, ctx in jobs:
            O, LSE = torch.full_like(Q, 9.0), torch.full(Q.shape[:3], 9.0, device=DEV)
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                f(Q, 0.1, cache, window, 4, n, O, LSE)
            got.append((O, LSE))
        torch.cuda.synchronize()
        for x, y in zip(out, got):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    for job in jobs:
        job[-1].close()


def test_far_pages():
    """Pages beyond 2^32 bytes of a pool."""
    ssb = _ssb()
    H_kv, d, page, n = 8, 128, 64, 40000
    K, V = (torch.zeros(n, H_kv, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.tensor([[39999, 7, 33333, 16385, 2]], dtype=torch.int32, device=DEV)
    g = _gen(0)
    for t in (K, V):
        t[table[0].long()] = torch.randn(5, H_kv, page, d, generator=g).bfloat16().to(DEV)
    cache = ssb.Cache16(K, V, table)
    Q = queries(g, 1, 8, 1, d)
    O, LSE = step(ssb, 16, cache, Q, [300], 150, 30)
    check(Q, O, LSE, keys_of(cache, H_kv, [300], 1, 150, 30), d ** -0.5, 16)


# ------------------------------------------------------------------ whole steps and rounds

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d,page,window,sinks", [(128, 16, 50, 4), (64, 0, 33, 0), (64, 24, 1000, 3)])
def test_a_request_from_prompt_to_rounds(bits, d, page, window, sinks):
    """Prompts in pieces, decoding, and rounds of drafted tokens of which some are accepted - rotated, appended and
    attended to by the calls as a layer makes them - against attention over everything in fp64."""
    ssb = _ssb()
    B, H_kv, G, T, room = 3, 2, 3, 5, 240
    H_q, rot = H_kv * G, d // 2
    g = _gen(d + page)
    freq = [1e4 ** (-2 * i / rot) for i in range(rot // 2)]
    table = ssb.Rope(freq)
    cache = make(ssb, bits, B, H_kv, d, page, room, 1)
    ctx = ssb.Context(B, H_q, H_kv, d, 40, 40, cache.desc.page_size * cache.desc.pages_per_req)
    append = ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append
    decode = ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window
    chunk = ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window
    lens = [0] * B

    def turned(x, b, tokens):
        """fp64 rotation of [H, n, d] rows, rounded to bf16 as the calls round it."""
        x = x.double().cpu().numpy()
        at = np.stack([np.asarray(tokens)] * len(freq), 1)
        y = np.stack([rope.rotate(h, at, freq)[0] for h in x])
        return torch.from_numpy(y).bfloat16().double().numpy()

    def agree(Q, O, LSE, keys):
        """The queries were rotated by the calls under test: an error of a bf16 step in Q changes a score by 2^-8 |q| |k|."""
        check(Q, O, LSE, keys, d ** -0.5, bits)

    # prompts of ragged lengths, in two pieces of 40
    total = [70, 41, 13]
    for lo in (0, 40):
        rows = [min(max(n - lo, 0), 40) for n in total]
        Q, K, V = queries(g, B, H_q, 40, d), queries(g, B, H_kv, 40, d, "bthd"), queries(g, B, H_kv, 40, d)
        off = list(lens)
        Qr = torch.zeros_like(Q)
        append(cache, K, V, table, None, Q, Qr, _i32(off), _i32(rows))
        lens = [a + b for a, b in zip(lens, rows)]
        for b in range(B):
            want = turned(Q[b, :, : rows[b]], b, off[b] + np.arange(rows[b])) if rows[b] else None
            if rows[b]:
                err = np.abs(Qr[b, :, : rows[b]].double().cpu().numpy() - want)
                assert (err <= 2.0 ** -7 * np.abs(want) + 1e-5).all()  # (a step where the two round apart)
    # decoding: one token at a time
    for _ in range(3):
        Q, K, V = queries(g, B, H_q, 1, d), queries(g, B, H_kv, 1, d), queries(g, B, H_kv, 1, d)
        append(cache, K, V, table, None, Q, Q, _i32(lens))
        lens = [n + 1 for n in lens]
        O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
        decode(Q, d ** -0.5, cache, window, sinks, _i32(lens), O, LSE)
        agree(Q, O, LSE, keys_of(cache, H_kv, lens, 1, window, sinks))
    # rounds: candidates rotated, attended to, the accepted ones (a prefix, or picked rows) appended as they are
    for k in range(3):
        Q, K, V = queries(g, B, H_q, T, d), queries(g, B, H_kv, T, d), queries(g, B, H_kv, T, d)
        Qr, Kr = torch.empty_like(Q), torch.empty_like(K)
        n = _i32(lens)
        ctx.ss_rope_rotate(table, Q, K, Qr, Kr, pos_off=n)
        for b in range(B):
            want = turned(K[b], b, lens[b] + np.arange(T))
            assert (np.abs(Kr[b].double().cpu().numpy() - want) <= 2.0 ** -7 * np.abs(want) + 1e-5).all()
        O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
        ctx.ss_verify_begin(Qr, d ** -0.5)
        chunk(cache, window, sinks, n)
        ctx.ss_verify_local(Kr, V)
        ctx.ss_verify_finalize(O, LSE)
        kl, vl = Kr.double().cpu().numpy(), V.double().cpu().numpy()
        agree(Qr, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks, None, False,
                                  lambda b, h, t: (kl[b, h, : t + 1], vl[b, h, : t + 1])))
        took = [(k + b) % (T + 1) for b in range(B)]
        append(cache, Kr, V, dst_off=n, row_cnt=_i32(took), row_idx=torch.arange(T, dtype=torch.int32, device=DEV).repeat(B, 1))
        for b in range(B):                                     # what joined is what was attended to
            if took[b] and bits == 16:
                hk, hv = history(cache, b, np.arange(lens[b], lens[b] + took[b]))
                assert np.array_equal(hk, kl[b, :, : took[b]]) and np.array_equal(hv, vl[b, :, : took[b]])
        lens = [a + b for a, b in zip(lens, took)]
    assert ctx.ss_poll_status() == (0, 0)
    ctx.close()


def test_room_and_queries_that_pass_31_bits_together_are_refused():
    ssb = _ssb()
    room = 2 ** 31 - 16384 - 64
    table = torch.zeros(1, room // 64, dtype=torch.int32, device=DEV)
    cache = ssb.Cache16.empty(1, 1, 64, 64, table)
    for T, fits in ((4, True), (40, False)):
        ctx = ssb.Context(1, 1, 1, 64, T, T, room)
        Q, O = (torch.ones(1, 1, T, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        call = lambda: ctx.ss_decode_window(Q, 1.0, cache, 2 ** 31 - 1, 2 ** 31 - 1, _i32([7]), O)
        if fits:
            call()
            assert ctx.ss_poll_status() == (0, 0) and not O.any()
        else:
            with pytest.raises(ssb.SpecStreamError) as e:
                call()
            assert e.value.status == ssb.SS_ERR_SHAPE
        ctx.close()


@pytest.mark.parametrize("bits", [16, 8])
def test_captured_behind_copies_and_other_kernels(bits):
    """A step and a round in one graph, each call right behind a copy or a kernel that writes what it reads."""
    ssb = _ssb()
    B, H_kv, G, d, T, room, window = 3, 2, 2, 64, 2, 320, 70
    g = _gen(17)
    cache, other = (make(ssb, bits, B, H_kv, d, 16, room, 3) for _ in range(2))
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, room)
    rope = ssb.Rope([1.0 / (i + 1) for i in range(d // 2)])
    src = [queries(g, B, h, T, d) for h in (H_kv * G, H_kv, H_kv)]
    buf = [torch.zeros_like(x) for x in src]
    lens = [_i32([5, 200, 0]), _i32([71, 90, 300])]
    here, n, after = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(3))
    out = [(torch.empty_like(src[0]), torch.empty(src[0].shape[:3], device=DEV)) for _ in range(4)]
    append = ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append
    decode = ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window
    chunk = ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window

    def run(c, a, b):
        n.copy_(here)
        append(c, buf[1], buf[2], rope, None, buf[0], buf[0], n)
        torch.add(n, T, out=after)
        decode(buf[0], 0.125, c, window, 3, after, *a)
        n.copy_(after)
        ctx.ss_verify_begin(buf[0], 0.125)
        chunk(c, window, 3, n)
        buf[1].copy_(src[1])
        ctx.ss_verify_local(buf[1], buf[2])
        ctx.ss_verify_finalize(*b)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run(cache, *out[:2])
        for k in (0, 1, 0):
            for c, go in ((cache, graph.replay), (other, lambda: run(other, *out[2:]))):
                here.copy_(lens[k])
                for x, y in zip(buf, src):
                    x.copy_(y)
                go()
            stream.synchronize()
            for x, y in zip(out[:2], out[2:]):
                assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
            for x, y in zip(cache.tensors, other.tensors):
                assert torch.equal(x, y)
            now = (lens[k] + T).tolist()
            local = lambda b, h, t: [x[b, h, :t + 1].double().cpu().numpy() for x in src[1:]]
            check(buf[0], *out[0], keys_of(cache, H_kv, now, T, window, 3), 0.125, bits)
            check(buf[0], *out[1], keys_of(cache, H_kv, now, T, window, 3, decode=False, local=local), 0.125, bits)
    assert ctx.ss_poll_status(stream) == (0, 0)
    ctx.close()
