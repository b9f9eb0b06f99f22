"""Rotary positions and rows that join a cache, on the GPU, against their definition in fp64."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8, rope
from tests.test_gpu_kv8 import make_cache, slots

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HOWS = {"bthd": (0, 2, 1, 3), "bhtd": (0, 1, 2, 3)}   # memory order of [B, H, T, d]


def _ssb():
    from paper_2609_33184_b200 import binding
    return binding


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rows(gen, shape, how="bhtd", pad=0):
    """Random bf16 rows of `shape` [B, H, T, d] laid out in another order, with `pad` spare elements behind a row."""
    order = HOWS[how]
    full = [shape[a] for a in order]
    full[-1] += pad
    t = torch.randn(full, generator=gen).bfloat16()[..., : shape[3]].to(DEV)
    return t.permute([order.index(a) for a in range(4)])


def _freq(rot, axes):
    n = rot // 2
    return [1e6 ** (-i / n) for i in range(n)], [i * axes // n for i in range(n)]


def _positions(gen, axes, B, T, far):
    top = 2 ** 31 - 1 if far else 1 << 17
    return torch.randint(-top - 1 if far else 0, top, (axes, B, T), generator=gen, dtype=torch.int64).to(torch.int32)


def _want(x, b, at, freq, inter, mag):
    """x [H, n, d] bf16 (CPU) -> fp64 rows and the sizes that errors scale with; at [n, pairs]."""
    H, n, d = x.shape
    out, size = zip(*(rope.rotate(x[h].double().numpy(), at, freq, inter, mag) for h in range(H)))
    return np.stack(out), np.stack(size)


def _close(got, want, size):
    """bf16 (half a step: 2^-8 of the value); in fp32 the angle off by 2^-23, sine and cosine by 2 units of 2^-24, the
    magnitude's product and the two products and their sum by 2^-24 each: below 2^-20 of the pair's length.  Elements that
    stay are bit for bit."""
    got = got.double().numpy()
    err = np.abs(got - want)
    assert (err <= 2.0 ** -8 * np.abs(want) * (size > 0) + 2.0 ** -20 * size).all(), float((err - 2.0 ** -8 * np.abs(want)).max())


def _at(pos, off, axis, b, rows):
    """[n, pairs] positions of rows of request b."""
    if pos is None:
        base = (0 if off is None else int(off[b])) + np.asarray(rows, dtype=np.int64)
        return np.stack([base] * len(axis), 1)
    return np.stack([pos[a, b].numpy().astype(np.int64)[rows] for a in axis], 1)


@pytest.mark.parametrize("d,rot,inter,axes,T,how", [
    (128, 128, False, 1, 8, "bhtd"), (128, 128, False, 3, 33, "bthd"), (128, 64, False, 1, 1, "bthd"), (128, 96, True, 3, 17, "bhtd"),
    (64, 64, False, 1, 5, "bthd"), (64, 16, False, 2, 64, "bhtd"), (64, 48, True, 4, 31, "bthd"), (64, 64, True, 1, 1, "bhtd"),
    (128, 16, True, 1, 400, "bthd"), (64, 32, False, 3, 900, "bhtd"),
])
@pytest.mark.parametrize("far", [False, True])
def test_rotate(d, rot, inter, axes, T, how, far):
    ssb = _ssb()
    B, H_q, H_kv, mag = 3, 6, 2, 1.0 if axes > 1 else 0.75
    g = _gen(d + rot + T + axes)
    Q, K = _rows(g, (B, H_q, T, d), how, 8), _rows(g, (B, H_kv, T, d), how)
    freq, axis = _freq(rot, axes)
    pos = _positions(g, axes, B, T, far)
    cnt = torch.tensor([T, T // 2, 0], dtype=torch.int32)
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    table = ssb.Rope(freq, axis, axes, inter, mag)
    Qo, Ko = torch.full_like(Q, 7.0), torch.full((B, T, H_kv, d), 7.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    ctx.ss_rope_rotate(table, Q, K, Qo, Ko, pos.to(DEV), row_cnt=cnt.to(DEV))
    assert ctx.ss_poll_status() == (0, 0)
    for x, y in ((Q.cpu(), Qo.cpu()), (K.cpu(), Ko.cpu())):
        for b in range(B):
            n = int(cnt[b])
            want, size = _want(x[b, :, :n], b, _at(pos, None, axis, b, np.arange(n)), freq, inter, mag)
            _close(y[b, :, :n], want, size)
            assert (y[b, :, n:] == 7.0).all()
    # in place, one of the two alone
    Q2 = Q.clone()
    ctx.ss_rope_rotate(table, Q2, None, Q2, None, pos.to(DEV), row_cnt=cnt.to(DEV))
    torch.cuda.synchronize()
    for b in range(B):
        n = int(cnt[b])
        assert torch.equal(Q2[b, :, :n], Qo[b, :, :n]) and torch.equal(Q2[b, :, n:], Q[b, :, n:])
    ctx.close()


@pytest.mark.parametrize("off", [None, [0, 131071, 2 ** 31 - 1 - 9]])
@pytest.mark.parametrize("axes", [1, 3])
def test_rotate_at_the_requests_positions(off, axes):
    """No positions: pos_off[b] + row on every axis; no counts: all rows."""
    ssb = _ssb()
    B, H_q, H_kv, d, T = 3, 4, 1, 128, 9
    g = _gen(5)
    Q, K = _rows(g, (B, H_q, T, d)), _rows(g, (B, H_kv, T, d))
    freq, axis = _freq(d, axes)
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    Qo, Ko = torch.empty_like(Q), torch.empty_like(K)
    ctx.ss_rope_rotate(ssb.Rope(freq, axis, axes), Q, K, Qo, Ko, pos_off=None if off is None else torch.tensor(off, dtype=torch.int32, device=DEV))
    assert ctx.ss_poll_status() == (0, 0)
    for x, y in ((Q.cpu(), Qo.cpu()), (K.cpu(), Ko.cpu())):
        for b in range(B):
            _close(y[b], *_want(x[b], b, _at(None, off, axis, b, np.arange(T)), freq, False, 1.0))
    ctx.close()


def _cache16(ssb, B, H_kv, d, page, room, seed, order=(0, 1, 2)):
    g = _gen(seed)
    per = -(-room // page) if page else 1
    shape = (B * per + 2, H_kv, page, d) if page else (B + 1, H_kv, room, d)
    K, V = (torch.randn([shape[a] for a in order] + [d], generator=g).bfloat16().to(DEV).permute([order.index(a) for a in range(3)] + [3])
            for _ in range(2))
    table = torch.randperm(shape[0], generator=g)[: B * per].view(B, per).to(torch.int32).to(DEV) if page else None
    return ssb.Cache16(K, V, table)


def _slots16(cache, b, tokens):
    K, _, table = cache.tensors
    tokens = np.asarray(tokens, dtype=np.int64)
    if table is None:
        return np.full_like(tokens, b), tokens
    return table[b].cpu().numpy()[tokens // K.shape[2]].astype(np.int64), tokens % K.shape[2]


@pytest.mark.parametrize("page,order", [(0, (0, 1, 2)), (1, (0, 1, 2)), (5, (0, 2, 1)), (16, (0, 1, 2)), (64, (0, 2, 1)), (256, (1, 0, 2))])
@pytest.mark.parametrize("d,rot,inter,axes,T", [(128, 128, False, 1, 1), (64, 32, True, 3, 7), (128, 96, False, 2, 200)])
@pytest.mark.parametrize("given", [False, True])
def test_append(page, order, d, rot, inter, axes, T, given):
    """Rows land where they belong, rotated; every other byte of the pools stays; the queries turn with them."""
    ssb = _ssb()
    B, H_q, H_kv = 4, 8, 2
    room = T + 90
    g = _gen(page + d + T)
    K, V, Q = _rows(g, (B, H_kv, T, d), "bthd"), _rows(g, (B, H_kv, T, d)), _rows(g, (B, H_q, T, d), "bthd", 16)
    freq, axis = _freq(rot, axes)
    pos = _positions(g, axes, B, T, False) if given else None
    off = torch.tensor([0, 90, 17, 3], dtype=torch.int32)
    cnt = torch.tensor([T, T, 0, (T + 1) // 2], dtype=torch.int32)
    cache = _cache16(ssb, B, H_kv, d, page, room, 3, order)
    before = [t.cpu().clone() for t in cache.tensors[:2]]
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    Qo = torch.full_like(Q, 7.0)
    ctx.ss_kv_append(cache, K, V, ssb.Rope(freq, axis, axes, inter), None if pos is None else pos.to(DEV), Q, Qo, off.to(DEV), cnt.to(DEV))
    assert ctx.ss_poll_status() == (0, 0)
    after = [t.cpu() for t in cache.tensors[:2]]
    touched = torch.zeros(after[0].shape[:1] + after[0].shape[2:3], dtype=torch.bool)
    for b in range(B):
        n = int(cnt[b])
        o, i = _slots16(cache, b, int(off[b]) + np.arange(n))
        touched[o, i] = True
        at = _at(pos, off, axis, b, np.arange(n))
        want, size = _want(K[b, :, :n].cpu(), b, at, freq, inter, 1.0)
        _close(after[0][o, :, i].transpose(0, 1), want, size)
        assert torch.equal(after[1][o, :, i].transpose(0, 1), V[b, :, :n].cpu())
        want, size = _want(Q[b, :, :n].cpu(), b, at, freq, inter, 1.0)
        _close(Qo[b, :, :n].cpu(), want, size)
        assert (Qo[b, :, n:] == 7.0).all()
    for x, y in zip(before, after):
        assert torch.equal(x.transpose(1, 2)[~touched], y.transpose(1, 2)[~touched])
    ctx.close()


@pytest.mark.parametrize("d,page,T", [(128, 16, 8), (64, 0, 3), (64, 1, 40), (128, 32, 1500)])
def test_append_of_accepted_rows_is_bit_exact(d, page, T):
    """Without a rotation: rows of a list, in its order, bit for bit (NaN and all); a row may be given twice."""
    ssb = _ssb()
    B, H_kv = 3, 2
    g = _gen(T)
    bits = lambda: torch.randint(-32768, 32767, (B, H_kv, T, d), generator=g, dtype=torch.int16).to(DEV).view(torch.bfloat16)
    K, V = bits(), bits()
    idx = torch.randint(0, T, (B, T), generator=g, dtype=torch.int32)
    cnt = torch.tensor([T, 1, 0], dtype=torch.int32)
    off = torch.tensor([2, 0, 5], dtype=torch.int32)
    cache = _cache16(ssb, B, H_kv, d, page, T + 8, 4)
    want = [t.view(torch.int16).cpu().clone() for t in cache.tensors[:2]]
    ctx = ssb.Context(B, H_kv, H_kv, d, 1, 1, 8)
    ctx.ss_kv_append(cache, K, V, dst_off=off.to(DEV), row_cnt=cnt.to(DEV), row_idx=idx.to(DEV))
    assert ctx.ss_poll_status() == (0, 0)
    for b in range(B):
        n = int(cnt[b])
        o, i = _slots16(cache, b, int(off[b]) + np.arange(n))
        for w, x in zip(want, (K, V)):
            w[o, :, i] = x.view(torch.int16).cpu()[b][:, idx[b, :n].long()].transpose(0, 1)
    for w, t in zip(want, cache.tensors):
        assert torch.equal(w, t.view(torch.int16).cpu())
    ctx.close()


@pytest.mark.parametrize("d,rot,inter,axes,T,page", [(128, 128, False, 1, 1, 16), (64, 32, True, 3, 9, 0), (128, 64, False, 1, 700, 24),
                                                     (64, 64, False, 2, 1300, 64), (64, 0, False, 1, 6, 8)])
@pytest.mark.parametrize("listed", [False, True])
def test_append_in_8_bits_is_rotate_then_write(d, rot, inter, axes, T, page, listed):
    ssb = _ssb()
    B, H_q, H_kv = 3, 6, 3
    g = _gen(d + T)
    K, V = _rows(g, (B, H_kv, T, d), "bthd"), _rows(g, (B, H_kv, T, d))
    K[0, 0, 0] = 0.0
    K[1, 1, 0, :3] = torch.tensor([float("inf"), -1.0, 2e30])
    V[2, 0, T - 1, 5] = float("nan")
    off = torch.tensor([4, 0, 11], dtype=torch.int32, device=DEV)
    cnt = torch.tensor([T, T, max(1, T // 3)], dtype=torch.int32, device=DEV)
    idx = torch.randint(0, T, (B, T), generator=g, dtype=torch.int32).to(DEV) if listed else None
    pos = _positions(g, axes, B, T, False).to(DEV) if rot else None
    table = ssb.Rope(*_freq(rot, axes), axes, inter) if rot else None
    one, two = (make_cache(ssb, B, H_kv, d, page, T + 20, 9, spare=2) for _ in range(2))
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    Kr = K.contiguous().clone()
    if rot:
        ctx.ss_rope_rotate(table, None, K, None, Kr, pos)
    ctx.ss_kv8_write(two, Kr, V, off, cnt, idx)
    Q = _rows(g, (B, H_q, T, d)) if rot and not listed else None
    Qo = None if Q is None else torch.zeros_like(Q)
    ctx.ss_kv8_append(one, K, V, table, pos, Q, Qo, off, cnt, idx)
    assert ctx.ss_poll_status() == (0, 0)
    for x, y, codes in zip(one.tensors[:4], two.tensors[:4], (True, True, False, False)):
        same = x == y
        if codes:                                              # a NaN's sign is free
            same |= ((x & 0x7F) == 0x7F) & ((y & 0x7F) == 0x7F)
        assert same.all()
    if Q is not None:
        want = torch.zeros_like(Q)
        ctx.ss_rope_rotate(table, Q, None, want, None, pos, row_cnt=cnt)
        torch.cuda.synchronize()
        assert torch.equal(Qo, want)
    ctx.close()


@pytest.mark.parametrize("bits", [16, 8])
def test_what_is_out_of_range_is_flagged_and_skipped(bits):
    ssb = _ssb()
    B, H_q, H_kv, d, T, page = 5, 2, 1, 64, 6, 16
    g = _gen(bits)
    K, V, Q = _rows(g, (B, H_kv, T, d)), _rows(g, (B, H_kv, T, d)), _rows(g, (B, H_q, T, d))
    cache = make_cache(ssb, B, H_kv, d, page, 32, 1) if bits == 8 else _cache16(ssb, B, H_kv, d, page, 32, 1)
    table = cache.tensors[-1]
    table[2, 0] = cache.tensors[0].shape[0]
    table[3, 1] = -1
    before = [t.cpu().clone() for t in cache.tensors[:-1]]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    off = i32(-2, 29, 3, 14, 2 ** 31 - 3)
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    append = ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append
    turn = ssb.Rope(*_freq(d, 1))
    Qo = torch.zeros_like(Q)
    append(cache, K, V, turn, None, Q, Qo, off)
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_DST_OVERFLOW | ssb.SS_DEV_BAD_PAGE)
    ok = {0: [0, 1, 2, 3], 1: [29, 30, 31], 3: [14, 15]}       # tokens that have a place
    live = torch.zeros(before[0].shape[0], page, dtype=torch.bool)
    for b, toks in ok.items():
        for t in toks:
            live[int(table[b, t // page]), t % page] = True
    changed = [(x.view(torch.uint8) != y.cpu().view(torch.uint8)).reshape(*x.shape[:3], -1).any(-1).any(1)
               for x, y in zip(before, cache.tensors)]
    assert torch.equal(changed[0], live) and torch.equal(changed[1], live)
    for c in changed[2:]:
        assert not (c & ~live).any()
    for b in range(4):                                         # (the last request's positions pass int32: turned in 64 bits)
        _close(Qo[b].cpu(), *_want(Q[b].cpu(), b, _at(None, off.cpu(), [0] * 32, b, np.arange(T)), _freq(d, 1)[0], False, 1.0))
    _close(Qo[4].cpu(), *_want(Q[4].cpu(), 4, _at(None, [0] * 4 + [2 ** 31 - 3], [0] * 32, 4, np.arange(T)), _freq(d, 1)[0], False, 1.0))
    # counts and row numbers
    append(cache, K, V, turn, None, None, None, i32(0, 0, 16, 0, 0), i32(-1, T + 3, 1, 1, 1), torch.full((B, T), T, dtype=torch.int32, device=DEV))
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_ACCEPT)
    ctx.close()


def test_refusals():
    ssb = _ssb()
    B, H_q, H_kv, d, T = 2, 4, 2, 64, 3
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    z = lambda H, T=T, d=d, B=B: torch.zeros(B, H, T, d, dtype=torch.bfloat16, device=DEV)
    Q, K, V = z(H_q), z(H_kv), z(H_kv)
    cache, cache8 = _cache16(ssb, B, H_kv, d, 8, 16, 0), make_cache(ssb, B, H_kv, d, 8, 16, 0)
    rot, wide = ssb.Rope(*_freq(64, 1)), ssb.Rope(*_freq(128, 1))
    pos = torch.zeros(1, B, T, dtype=torch.int32, device=DEV)

    def refused(status, f, *a, **k):
        with pytest.raises(ssb.SpecStreamError) as e:
            f(*a, **k)
        assert e.value.status == status

    refused(ssb.SS_ERR_SHAPE, ctx.ss_rope_rotate, wide, Q, K, Q, K)                   # more turns than the head has
    refused(ssb.SS_ERR_SHAPE, ctx.ss_rope_rotate, rot, z(H_q, B=3), None, z(H_q, B=3), None)
    for append, c in ((ctx.ss_kv_append, cache), (ctx.ss_kv8_append, cache8)):
        refused(ssb.SS_ERR_ARG, append, c, K, V, None, None, Q, Q)                    # queries without a rotation
        refused(ssb.SS_ERR_ARG, append, c, K, V, None, pos)                           # positions without one
        refused(ssb.SS_ERR_ARG, append, c, K, V, rot, None, Q, Q, row_idx=torch.zeros(B, T, dtype=torch.int32, device=DEV))
        refused(ssb.SS_ERR_SHAPE, append, c, K, V, wide)
    odd = torch.zeros(B, H_kv, T, d + 4, dtype=torch.bfloat16, device=DEV)[..., :d]   # rows 8 bytes off
    refused(ssb.SS_ERR_ALIGN, ctx.ss_kv_append, cache, odd, V, rot)
    refused(ssb.SS_ERR_ALIGN, ctx.ss_kv_append, cache, K, odd, rot)
    refused(ssb.SS_ERR_ALIGN, ctx.ss_rope_rotate, rot, None, odd, None, K)
    refused(ssb.SS_ERR_ALIGN, ctx.ss_rope_rotate, rot, None, K, None, odd)
    for bad in (lambda: ctx.ss_kv_append(cache8, K, V, rot), lambda: ctx.ss_kv8_append(cache, K, V, rot),
                lambda: ctx.ss_rope_rotate(rot, Q.float(), None, Q, None), lambda: ctx.ss_rope_rotate(rot, Q, None, K, None),
                lambda: ctx.ss_rope_rotate(rot, Q.cpu(), None, Q, None), lambda: ctx.ss_rope_rotate(rot, Q, K, Q, K, pos[:, :1]),
                lambda: ctx.ss_rope_rotate(rot, Q, K, Q, K, pos.long()), lambda: ctx.ss_rope_rotate(rot, None, K, Q, K),
                lambda: ctx.ss_kv_append(cache, z(H_kv, d=128), V, rot)):
        with pytest.raises(AssertionError):
            bad()
    assert ctx.ss_poll_status() == (0, 0)
    # the C entry points' own checks
    no, t = ssb.ss_tensor(None, 0, 0, 0), ssb.as_ss_tensor
    L, h = ctx.lib, ctx.handle
    assert L.ss_rope_rotate(h, None, t(Q), t(K), B, T, None, None, None, t(Q), t(K), None) == ssb.SS_ERR_ARG
    assert L.ss_rope_rotate(h, rot.ref, no, no, B, T, None, None, None, no, no, None) == ssb.SS_ERR_ARG
    assert L.ss_rope_rotate(h, rot.ref, t(Q), no, B, T, None, None, None, no, no, None) == ssb.SS_ERR_ARG
    assert L.ss_rope_rotate(h, rot.ref, t(Q), no, B, 0, None, None, None, t(Q), no, None) == ssb.SS_ERR_ARG
    assert L.ss_rope_rotate(h, rot.ref, t(Q), no, B, 1 << 29, None, None, None, t(Q), no, None) == ssb.SS_ERR_SHAPE
    assert L.ss_rope_rotate(h, rot.ref, t(Q), no, B, T, pos.data_ptr() + 2, None, None, t(Q), no, None) == ssb.SS_ERR_ALIGN
    assert L.ss_kv_append(h, None, t(K), t(V), B, T, None, None, None, None, None, no, no, None) == ssb.SS_ERR_ARG
    assert L.ss_kv_append(h, cache.ref, no, t(V), B, T, None, None, None, None, None, no, no, None) == ssb.SS_ERR_ARG
    junk = ssb.ss_rope()
    C.memmove(C.byref(junk), rot.ref, C.sizeof(junk))
    junk.rot_dim = 24
    assert L.ss_rope_rotate(h, C.byref(junk), t(Q), no, B, T, None, None, None, t(Q), no, None) == ssb.SS_ERR_SHAPE
    ctx.close()


def test_far_pages():
    """Places beyond 2^32 bytes of a pool."""
    ssb = _ssb()
    H_kv, d, page, n = 8, 128, 64, 40000                       # 131,072 bytes a page
    K, V = (torch.empty(n, H_kv, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.tensor([[39999, 7], [16385, 32769]], dtype=torch.int32, device=DEV)
    g = _gen(0)
    x, y = _rows(g, (2, H_kv, 3, d)), _rows(g, (2, H_kv, 3, d))
    ctx = ssb.Context(2, H_kv, H_kv, d, 1, 1, 8)
    ctx.ss_kv_append(ssb.Cache16(K, V, table), x, y, dst_off=torch.tensor([62, 63], dtype=torch.int32, device=DEV))
    assert ctx.ss_poll_status() == (0, 0)
    for b, places in enumerate((((39999, 62), (39999, 63), (7, 0)), ((16385, 63), (32769, 0), (32769, 1)))):
        for k, (o, i) in enumerate(places):
            assert torch.equal(K[o, :, i], x[b, :, k]) and torch.equal(V[o, :, i], y[b, :, k])
    ctx.close()


def test_captured_on_another_stream():
    """A captured step follows offsets, counts and positions that change between replays."""
    ssb = _ssb()
    B, H_q, H_kv, d, T = 2, 4, 2, 128, 2
    g = _gen(8)
    K, V, Q = _rows(g, (B, H_kv, T, d)), _rows(g, (B, H_kv, T, d)), _rows(g, (B, H_q, T, d))
    cache, plain = (_cache16(ssb, B, H_kv, d, 8, 64, 2) for _ in range(2))
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    rot = ssb.Rope(*_freq(d, 1))
    off = torch.zeros(B, dtype=torch.int32, device=DEV)
    Qo, Qw = torch.zeros_like(Q), torch.zeros_like(Q)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.ss_kv_append(cache, K, V, rot, None, Q, Qo, off)
        for step in range(5):
            off.copy_(torch.tensor([2 * step, 50 - 7 * step], dtype=torch.int32))
            graph.replay()
            ctx.ss_kv_append(plain, K, V, rot, None, Q, Qw, off, stream=stream)
            stream.synchronize()
            assert torch.equal(Qo, Qw)
            for x, y in zip(cache.tensors, plain.tensors):
                assert torch.equal(x, y)
    assert ctx.ss_poll_status(stream) == (0, 0)
    ctx.close()


@pytest.mark.parametrize("d,H_q,H_kv,rot,inter,axes", [(128, 4, 1, 128, False, 1), (64, 3, 1, 32, True, 3), (128, 8, 2, 64, False, 2), (64, 2, 2, 64, True, 1)])
@pytest.mark.parametrize("bits,listed", [(0, False), (16, False), (16, True), (8, False), (8, True)])
def test_a_large_call_is_many_small_ones(bits, listed, d, H_q, H_kv, rot, inter, axes):
    """The same bits, whichever way rows are dealt to threads; ragged, with and without Q, rows in order and by a list."""
    ssb = _ssb()
    B, T, piece = 3, 4007, 200
    g = _gen(d + H_q + bits)
    Q, K, V = (_rows(g, (B, h, T, d), "bthd") for h in (H_q, H_kv, H_kv))
    freq, axis = _freq(rot, axes)
    rope = ssb.Rope(freq, axis, axes, inter, 1.25)
    pos = _positions(g, axes, B, T, True)
    cnt, off = torch.tensor([T, 1300, T - 7], dtype=torch.int32), torch.tensor([0, 100, 5], dtype=torch.int32)
    idx = torch.stack([torch.randperm(T, generator=g) for _ in range(B)]) if listed else None
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 8)
    caches = [None, None]
    if bits == 16:
        caches = [_cache16(ssb, B, H_kv, d, 16, 4128, 3) for _ in range(2)]
    elif bits == 8:
        table = torch.arange(3 * 258, dtype=torch.int32, device=DEV).view(3, 258)
        caches = [ssb.Cache8.empty(3 * 258, H_kv, 16, d, table) for _ in range(2)]

    def call(cache, Q, K, V, Qo, Ko, pos, off, cnt, idx):
        pos, off, cnt = (x.contiguous().to(DEV) for x in (pos, off, cnt))
        if cache is None:
            ctx.ss_rope_rotate(rope, Q, K, Qo, Ko, pos, row_cnt=cnt)
        else:
            idx = None if idx is None else idx.to(torch.int32).to(DEV)
            (ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append)(cache, K, V, rope, pos, Q, Qo, off, cnt, idx)

    outs = [(None if listed else torch.full_like(Q, 7.0), torch.full_like(K, 7.0)) for _ in range(2)]
    call(caches[0], None if listed else Q, K, V, *outs[0], pos, off, cnt, idx)
    if listed:   # the listed rows, in order
        rows = idx.to(DEV)[:, None, :, None].expand(B, H_kv, T, d)
        K, V = K.gather(2, rows), V.gather(2, rows)
        pos = pos.gather(2, idx[None].expand(axes, B, T))
    for s in range(0, T, piece):
        e = min(s + piece, T)
        cut = lambda x: None if x is None else x[:, :, s:e]
        call(caches[1], None if listed else cut(Q), cut(K), cut(V), cut(outs[1][0]), cut(outs[1][1]), cut(pos), off + s,
             (cnt - s).clamp(0, e - s), None)
    assert ctx.ss_poll_status() == (0, 0)
    for x, y in zip(outs[0], outs[1]):
        assert x is None or torch.equal(x, y)
    if bits:
        for x, y in zip(caches[0].tensors, caches[1].tensors):
            assert torch.equal(x, y)
    if not listed:
        for b in range(B):
            n = int(cnt[b])
            some = torch.randperm(n, generator=g)[:50].numpy()
            want, size = _want(Q[b].cpu()[:, some], b, _at(pos, None, axis, b, some), freq, inter, 1.25)
            _close(outs[0][0][b].cpu()[:, some], want, size)
    ctx.close()


@pytest.mark.parametrize("T", [1, 3, 11])
@pytest.mark.parametrize("d,H_q,H_kv,bits", [(128, 16, 4, 16), (128, 16, 4, 8), (64, 40, 8, 0), (64, 4, 1, 8), (128, 3, 1, 16)])
def test_many_requests_of_few_tokens(d, H_q, H_kv, bits, T):
    """Enough requests for a large call, rows of several heads side by side in a block: the bits of calls of a few requests."""
    ssb = _ssb()
    B, room = 60 + 80000 * d // 64 // (H_q + 2 * H_kv) // T, 16
    g = _gen(T + d)
    Q, K, V = (_rows(g, (B, h, T, d)) for h in (H_q, H_kv, H_kv))
    rope = ssb.Rope(*_freq(d, 2), 2, False)
    pos = _positions(g, 2, B, T, True).to(DEV)
    cnt, off = (torch.randint(0, top, (B,), generator=g, dtype=torch.int32).to(DEV) for top in (T + 1, room + 1 - T))
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, room)
    kind = {16: ssb.Cache16, 8: ssb.Cache8}.get(bits)
    caches = [kind.empty(B, H_kv, room, d) for _ in range(2)] if bits else [None, None]
    outs = [(torch.full_like(Q, 7.0), torch.full_like(K, 7.0)) for _ in range(2)]

    def call(cache, out, at):
        Qs, Ks, Vs, Qo, Ko, ps = Q[at], K[at], V[at], out[0][at], out[1][at], pos[:, at].contiguous()
        if not bits:
            ctx.ss_rope_rotate(rope, Qs, Ks, Qo, Ko, ps, row_cnt=cnt[at])
        else:
            part = kind(*(x[at] for x in cache.tensors[:-1]))
            (ctx.ss_kv8_append if bits == 8 else ctx.ss_kv_append)(part, Ks, Vs, rope, ps, Qs, Qo, off[at], cnt[at])

    call(caches[0], outs[0], slice(0, B))
    for s in range(0, B, B // 9):
        call(caches[1], outs[1], slice(s, min(s + B // 9, B)))
    assert ctx.ss_poll_status() == (0, 0)
    for x, y in zip(outs[0], outs[1]):
        assert torch.equal(x, y)
    if bits:
        for x, y in zip(caches[0].tensors[:-1], caches[1].tensors[:-1]):
            assert torch.equal(x, y)
    live = (torch.arange(T, device=DEV)[None] < cnt[:, None])[:, None, :, None].expand_as(Q)
    assert (outs[0][0][~live] == 7.0).all()
    b = int(cnt.argmax())
    n = int(cnt[b])
    if n:
        _close(outs[0][0][b, :, :n].cpu(), *_want(Q[b].cpu()[:, :n], b, _at(pos.cpu(), None, _freq(d, 2)[1], b, np.arange(n)), _freq(d, 2)[0], False, 1.0))
    ctx.close()
