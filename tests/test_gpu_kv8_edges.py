"""The 8-bit KV cache on the GPU where its inputs leave the ordinary: rows that nobody wrote, scale bytes outside the
format."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8
from tests.test_gpu_kv8 import DEV, _gen, _ssb, check_attention, decode, history, make_cache, slots

pytestmark = pytest.mark.gpu


def whole_round(ctx, cache, Q, vl, scale, K_loc, V_loc):
    O = torch.full(Q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    LSE = torch.full(Q.shape[:3], float("nan"), device=DEV)
    ctx.ss_verify_begin(Q, scale)
    ctx.ss_verify_chunk8(cache, vl)
    ctx.ss_verify_local(K_loc, V_loc)
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (0, 0)
    return O, LSE


@pytest.mark.parametrize("flags", [0, 1], ids=["auto", "simt"])
@pytest.mark.parametrize("fill", ["empty", "zeros"])
@pytest.mark.parametrize("d", [64, 128])
def test_visible_tokens_that_were_never_written(d, fill, flags):
    """They are rows of zeros: score 0, value 0, in the row sum with weight e^0.  One request with none written, one with
    a few, whose scores differ from 0 by several binades, and long enough to be cut."""
    ssb = _ssb()
    B, H_q, H_kv, T, page, lens = 3, 8, 2, 2, 16, [300, 2000, 1]
    per = 128
    cache = ssb.Cache8.empty(B * per, H_kv, page, d,
                             torch.randperm(B * per, generator=_gen(1)).to(torch.int32).view(B, per).to(DEV))
    if fill == "zeros":                        # a user's own buffers
        for t in cache.tensors[2:4]:
            t.zero_()
    g = _gen(d)
    K, V = (torch.randn(B, H_kv, 70, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    Q = torch.randn(B, H_q, T, d, generator=g).bfloat16().to(DEV)
    K_loc, V_loc = (torch.randn(B, H_kv, T, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    scale = 4 * d ** -0.5                       # scores of the written tokens up to about 16
    ctx = ssb.Context(B, H_q, H_kv, d, T, T, per * page, flags=flags)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    ctx.ss_kv8_write(cache, K, V, i32(0, 777, 0), i32(0, 70, 0))
    written = (torch.zeros(B, H_kv, 70, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    Kr, Vr = written
    ctx.ss_kv8_read(cache, Kr, Vr, i32(0, 777, 0), i32(70, 70, 70))
    assert (Kr[0] == 0).all() and (Vr[2] == 0).all()

    def kv(b):
        k, v = np.zeros((2, H_kv, lens[b], d))
        if b == 1:
            k[:, 777:847], v[:, 777:847] = Kr[1].double().cpu().numpy(), Vr[1].double().cpu().numpy()
        return k, v
    O, LSE = decode(ssb, cache, Q, lens, scale=scale, ctx=ctx)
    assert ctx.last_chunk_kernel() == ("kv8-simt" if flags else "kv8-tcgen05")
    check_attention(Q, O, LSE, kv, scale)
    assert (O[0] == 0).all()
    O, LSE = whole_round(ctx, cache, Q, i32(*lens), scale, K_loc, V_loc)
    f = lambda t, b, n: t[b, :, :n].double().cpu().numpy()
    for i in range(T):
        near = lambda b: (np.concatenate([kv(b)[0], f(K_loc, b, i + 1)], 1), np.concatenate([kv(b)[1], f(V_loc, b, i + 1)], 1))
        check_attention(Q[:, :, i:i + 1], O[:, :, i:i + 1], LSE[:, :, i:i + 1], near, scale)
    ctx.close()


@pytest.mark.parametrize("flags", [0, 1], ids=["auto", "simt"])
@pytest.mark.parametrize("d", [64, 128])
def test_scale_bytes_outside_the_format_count_as_its_ends(d, flags):
    """Bytes below 95 as 95, above 207 as 207, in attention and in reading back."""
    ssb = _ssb()
    B, H_q, H_kv, n = 2, 8, 2, 700
    cache = make_cache(ssb, B, H_kv, d, 32, n, 9)
    K, V, Ks, Vs, _ = cache.tensors
    pick = lambda shape, bytes_, seed: torch.tensor(bytes_, dtype=torch.uint8)[
        torch.randint(0, len(bytes_), shape, generator=_gen(seed))].to(DEV)
    Ks.copy_(pick(Ks.shape, [0, 1, 94, 95, 118, 119], 1))
    Vs.copy_(pick(Vs.shape, [0, 94, 95, 120, 200, 206, 207, 208, 254, 255], 2))

    def clamped(b):
        out = []
        for k in (0, 1):
            o, i = slots(cache, b, np.arange(n))
            byte = np.clip(cache.tensors[2 + k].cpu().numpy()[o, :, i], 95, 207)
            codes = cache.tensors[k].cpu().numpy()[o, :, i]
            out.append((kv8.VALUES[codes] * np.exp2(byte.astype(np.float64) - 127.0)[..., None]).transpose(1, 0, 2))
        return out
    Q = torch.randn(B, H_q, 1, d, generator=_gen(3)).bfloat16().to(DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 1024, flags=flags)
    Kr, Vr = (torch.empty(B, H_kv, n, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.ss_kv8_read(cache, Vr, Kr)
    ctx.ss_kv8_read(cache, Kr, Vr)
    for b in range(B):
        k, v = clamped(b)
        assert np.array_equal(Kr[b].double().cpu().numpy(), k) and np.array_equal(Vr[b].double().cpu().numpy(), v)
        hk, hv = history(cache, b, n)           # and so the oracle reads them
        assert np.array_equal(hk, k) and np.array_equal(hv, v)
    O, LSE = decode(ssb, cache, Q, [n, 130], ctx=ctx)
    check_attention(Q, O, LSE, lambda b: [x[:, :[n, 130][b]] for x in clamped(b)], d ** -0.5)
    ctx.close()


@pytest.mark.parametrize("first", ["chunk8", "chunk"])
def test_rows_read_back_inside_a_round_are_the_next_call_s_history(first):
    """Under overlapped launches: a chunk of any kind, ss_kv8_read into a buffer, that buffer as the next chunk, another
    read, its rows as the local segment."""
    ssb = _ssb()
    B, H_q, H_kv, d, T, n, T_loc = 8, 16, 8, 128, 4, 4096, 512
    small, big = (make_cache(ssb, B, H_kv, d, page, room, seed) for page, room, seed in ((16, 256, 1), (64, n, 2)))
    g = _gen(7)
    Q = torch.randn(B, H_q, T, d, generator=g).bfloat16().to(DEV)
    K0, V0 = (torch.randn(B, H_kv, 256, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    K, V = (torch.empty(B, H_kv, n, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    Kl, Vl = (torch.empty(B, H_kv, T_loc, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    off = torch.full((B,), n - T_loc, dtype=torch.int32, device=DEV)
    O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, T, T_loc, n, flags=ssb.SS_FLAG_OVERLAP_CHUNKS)
    results = []
    for _ in range(20):
        for t in (K, V, Kl, Vl):
            t.zero_()
        ctx.ss_verify_begin(Q, d ** -0.5)
        if first == "chunk8":
            ctx.ss_verify_chunk8(small)
        else:
            ctx.ss_verify_chunk(K0, V0)
        ctx.ss_kv8_read(big, K, V)
        ctx.ss_verify_chunk(K, V)
        ctx.ss_kv8_read(big, Kl, Vl, src_off=off)
        ctx.ss_verify_local(Kl, Vl)
        ctx.ss_verify_finalize(O, LSE)
        results.append((O.clone(), LSE.clone()))
    assert ctx.ss_poll_status() == (0, 0)
    f = lambda t, b: t[b].double().cpu().numpy()

    def kv(b, i):
        k, v = history(big, b, n)
        a = history(small, b, 256) if first == "chunk8" else [f(K0, b), f(V0, b)]
        seen = slice(n - T_loc, n - T + i + 1)
        return np.concatenate([a[0], k, k[:, seen]], 1), np.concatenate([a[1], v, v[:, seen]], 1)
    for i in range(0, T, 3):
        check_attention(Q[:1, :, i:i + 1], results[0][0][:1, :, i:i + 1], results[0][1][:1, :, i:i + 1], lambda b: kv(b, i),
                        d ** -0.5)
    for o, l in results[1:]:
        assert torch.equal(o, results[0][0]) and torch.equal(l, results[0][1])
    ctx.close()


@pytest.mark.parametrize("page,kernel", [(24, "kv8-simt"), (16, "kv8-tcgen05")])
@pytest.mark.parametrize("value", ["inf", "-inf", "nan"])
def test_a_query_that_is_not_finite_makes_its_row_nan_on_both_kernels(page, kernel, value):
    """Also where every product with it has the same sign, so that all scores would be -inf or all inf."""
    ssb = _ssb()
    B, H_q, H_kv, d, T, n = 1, 4, 2, 64, 2, 500
    cache = make_cache(ssb, B, H_kv, d, page, n, 3)
    K = cache.tensors[0]
    K[..., 7] = (K[..., 7] & 0x7F) | 0x08       # positive, not zero (and no NaN: make_cache has none)
    K[..., 7] = torch.where(K[..., 7] == 0x7F, torch.full_like(K[..., 7], 0x30), K[..., 7])
    Q = torch.randn(B, H_q, T, d, generator=_gen(1)).bfloat16().to(DEV)
    bad = Q.clone()
    bad[0, 1, 0, 7], bad[0, 2, 1, 7] = float(value), float(value)
    hit = torch.zeros(B, H_q, T, dtype=torch.bool, device=DEV)
    hit[0, 1, 0] = hit[0, 2, 1] = True
    ctx = ssb.Context(B, H_q, H_kv, d, T, T, 1024)
    good, gl = decode(ssb, cache, Q, [n], ctx=ctx)
    O, LSE = decode(ssb, cache, bad, [n], ctx=ctx)
    assert ctx.last_chunk_kernel() == kernel
    assert torch.isnan(O[hit]).all() and torch.isnan(LSE[hit]).all()
    assert torch.equal(O[~hit], good[~hit]) and torch.equal(LSE[~hit], gl[~hit])
    if page == 24:                              # with every page outside the pool the row is NaN all the same
        table = cache.tensors[4].clone()
        cache.tensors[4].fill_(-1)
        vl = torch.tensor([n], dtype=torch.int32, device=DEV)
        ctx.ss_decode8(bad, d ** -0.5, cache, vl, O, LSE)
        assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_PAGE)
        assert torch.isnan(O[hit]).all() and torch.isnan(LSE[hit]).all() and (O[~hit] == 0).all()
        cache.tensors[4].copy_(table)
    ctx.close()


@pytest.mark.parametrize("what", ["two", "bf16", "fold", "export", "one"])
@pytest.mark.parametrize("page", [16, 24])
def test_nan_rows_pass_through_every_merge(what, page):
    """A row made NaN by its query or by a NaN in a visible key stays NaN, O and LSE, whatever its states are
    merged with and on whichever path; the other rows come out as without it."""
    ssb = _ssb()
    B, H_q, H_kv, d, T, lens = 2, 8, 2, 128, 3, [900, 140]
    caches = [make_cache(ssb, B, H_kv, d, page, 912, 4 + k) for k in range(2)]
    g = _gen(2)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)
    Q, K, V, K_loc, V_loc = rnd(B, H_q, T, d), rnd(B, H_kv, 128, d), rnd(B, H_kv, 128, d), rnd(B, H_kv, T, d), rnd(B, H_kv, T, d)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, T, T, 1024, max_chunks=2 if what == "fold" else 8)

    def run(Q):
        O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
        ctx.ss_verify_begin(Q, d ** -0.5)
        ctx.ss_verify_chunk8(caches[0], vl)
        if what in ("two", "fold"):
            for k in (1, 0, 1):
                ctx.ss_verify_chunk8(caches[k], vl)
        elif what == "bf16":
            ctx.ss_verify_chunk(K, V)
        elif what == "export":
            ml, a = torch.empty(B * H_q * T, 2, device=DEV), torch.empty(B * H_q * T, d, device=DEV)
            ctx.ss_verify_export_state(ml, a)
            ctx.ss_verify_abort()
            ctx.ss_verify_begin(Q, d ** -0.5)
            ctx.ss_verify_import_state(ml, a)
        ctx.ss_verify_local(K_loc, V_loc)
        ctx.ss_verify_finalize(O, LSE)
        assert ctx.ss_poll_status() == (0, 0)
        return O, LSE
    good, gl = run(Q)
    assert torch.isfinite(good).all() and torch.isfinite(gl).all()
    bad = Q.clone()
    hit = torch.zeros(B, H_q, T, dtype=torch.bool, device=DEV)
    for i, (b, h, t) in enumerate([(0, 1, 0), (0, 6, 2), (1, 7, 1), (1, 0, 0)]):
        bad[b, h, t, 5 * i] = [float("nan"), float("inf"), float("-inf"), float("nan")][i]
        hit[b, h, t] = True
    O, LSE = run(bad)
    assert torch.isnan(O[hit]).all() and torch.isnan(LSE[hit]).all()
    assert torch.equal(O[~hit], good[~hit]) and torch.equal(LSE[~hit], gl[~hit])
    # one NaN code in a key of the second request's second head: all rows of that head
    o, i = slots(caches[0], 1, [77])
    caches[0].tensors[0][int(o[0]), 1, int(i[0]), 9] = 0x7F
    O, LSE = run(Q)
    hit.zero_()
    hit[1, 4:] = True
    assert torch.isnan(O[hit]).all() and torch.isnan(LSE[hit]).all()
    assert torch.equal(O[~hit], good[~hit]) and torch.equal(LSE[~hit], gl[~hit])
    ctx.close()
