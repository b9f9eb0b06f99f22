"""The 8-bit KV cache on the GPU: writing, reading back and attention against fp64."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import kv8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ssb():
    from paper_2609_33184_b200 import binding
    return binding


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _strided(shape, order, dtype, gen, pad):
    """A tensor of `shape` [outer, H, T, ..] laid out in `order` of its first three axes, with `pad` spare
    elements behind every row, filled with random bytes."""
    full = [shape[a] for a in order] + [s for s in shape[3:]]
    if len(shape) == 4:
        full[-1] += pad
    n = math.prod(full)
    t = torch.randint(0, 255, (n,), generator=gen, dtype=torch.uint8).to(DEV).view(dtype).view(full)
    if len(shape) == 4:
        t = t[..., : shape[3]]
    inv = [order.index(a) for a in range(3)] + list(range(3, len(shape)))
    return t.permute(inv)


def make_cache(ssb, B, H_kv, d, page, room, seed, order=(0, 1, 2), pad=0, spare=2):
    """A cache with random contents: page 0 = dense."""
    g = _gen(seed)
    per = -(-room // page) if page else 1
    outer, tokens = (B * per + spare, page) if page else (B + spare, room)
    K, V = (_strided((outer, H_kv, tokens, d), list(order), torch.uint8, g, pad) for _ in range(2))
    Ks, Vs = (_strided((outer, H_kv, tokens), list(order), torch.uint8, g, 0) for _ in range(2))
    Ks.copy_(Ks % 7 + 116)
    Vs.copy_(Vs % 9 + 112)
    table = None
    if page:
        table = torch.randperm(outer, generator=g)[: B * per].view(B, per).to(torch.int32).to(DEV)
    for t in (K, V):                          # no NaN codes but where a test puts them
        t.copy_(torch.where((t & 0x7F) == 0x7F, torch.zeros_like(t), t))
    return ssb.Cache8(K, V, Ks, Vs, table)


def slots(cache, b, tokens):
    """(outer, inner) of tokens of request b."""
    K, table = cache.tensors[0], cache.tensors[4]
    tokens = np.asarray(tokens, dtype=np.int64)
    if table is None:
        return np.full_like(tokens, b), tokens
    page = K.shape[2]
    return table[b].cpu().numpy()[tokens // page].astype(np.int64), tokens % page


def history(cache, b, n):
    """fp64 K, V [H_kv, n, d] of request b's first n tokens."""
    o, i = slots(cache, b, np.arange(n))
    out = []
    for k in (0, 1):
        codes = cache.tensors[k].cpu().numpy()[o, :, i]
        byte = cache.tensors[2 + k].cpu().numpy()[o, :, i]
        out.append(kv8.decode(codes, byte).transpose(1, 0, 2).reshape(codes.shape[1], n, codes.shape[2]))
    return out


def poison(cache, lens):
    """NaN codes and scale bytes 255 behind every request's last token, page ids from the first unused page on."""
    K, V, Ks, Vs, table = cache.tensors
    room = K.shape[2] * (1 if table is None else table.shape[1])
    for b, n in enumerate(lens):
        o, i = slots(cache, b, np.arange(n, room))
        o, i = torch.as_tensor(o, device=DEV), torch.as_tensor(i, device=DEV)
        K[o, :, i], V[o, :, i], Ks[o, :, i], Vs[o, :, i] = 0x7F, 0xFF, 255, 255
        if table is not None:
            table[b, -(-n // K.shape[2]):] = -7


def check_attention(Q, O, LSE, ref_kv, scale):
    """ref_kv(b) -> K, V [H_kv, n, d] fp64.  Tolerances: O is bf16 (half a step: 2^-8 of the value); a weight is
    off by at most 2^-9 of itself where it is held in 16 bits or as three short terms, and by 2^-30 of the largest
    weight where those underflow; scores and exponentials in fp32 add below 2^-14 (d products, |score| < 2^7).
    A = sum p|v| carries the relative errors, n * 2^-30 * max|v| the absolute ones."""
    B, H_q, T, d = Q.shape
    q = Q.double().cpu().numpy()
    Og, Lg = O.double().cpu().numpy(), LSE.double().cpu().numpy()
    for b in range(B):
        K, V = ref_kv(b)
        G = H_q // K.shape[0]
        for h in range(K.shape[0]):
            n = K.shape[1]
            o, lse, A = kv8.attention(q[b, h * G:(h + 1) * G].reshape(G * T, d), K[h], V[h], scale)
            og, lg = Og[b, h * G:(h + 1) * G].reshape(G * T, d), Lg[b, h * G:(h + 1) * G].reshape(-1)
            if n == 0:
                assert (og == 0).all() and (lg == -np.inf).all()
                continue
            vmax = np.abs(V[h]).max()
            tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -9 + 2.0 ** -13) * A + n * 2.0 ** -30 * vmax + 1e-30
            assert np.isfinite(og).all(), (b, h)
            bad = np.abs(og - o) / tol
            assert bad.max() <= 1.0, (b, h, float(bad.max()))
            # d products of |q k| in fp32, each partial sum off by 2^-23 of it, and the sum of the weights; query
            # values below 2^-13 of their row's maximum may be off by 2^-17 of that maximum
            qr = q[b, h * G:(h + 1) * G].reshape(G * T, d)
            s_abs = scale * (np.abs(qr) @ np.abs(K[h]).T).max(1)
            top = np.abs(qr).max(1, keepdims=True)
            low = scale * 2.0 ** -17 * ((np.abs(qr) < 2.0 ** -13 * top) * top) @ np.abs(K[h]).T
            ltol = 2.0 ** -18 * s_abs + 2.0 ** -20 * np.abs(lse) + 2.0 ** -16 + low.max(1)
            assert (np.abs(lg - lse) <= ltol).all(), (b, h, float(np.abs(lg - lse).max()))


def decode(ssb, cache, Q, lens, scale=None, ctx=None, stream=None):
    B, H_q, T, d = Q.shape
    own = ctx is None
    room = cache.desc.page_size * cache.desc.pages_per_req
    ctx = ctx or ssb.Context(B, H_q, cache.H_kv, d, T, 1, room)
    vl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    O = torch.full((B, H_q, T, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    LSE = torch.full((B, H_q, T), float("nan"), device=DEV)
    ctx.ss_decode8(Q, scale or d ** -0.5, cache, vl, O, LSE, stream)
    torch.cuda.synchronize()
    assert ctx.ss_poll_status() == (0, 0)
    if own:
        ctx.close()
    return O, LSE


# ------------------------------------------------------------------ writing and reading

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,order,pad", [(0, (0, 1, 2), 0), (1, (0, 1, 2), 16), (5, (0, 2, 1), 0), (16, (0, 1, 2), 0),
                                            (64, (0, 2, 1), 32), (128, (1, 0, 2), 0)])
def test_write_is_bit_exact_and_touches_nothing_else(d, page, order, pad):
    ssb = _ssb()
    B, H_kv, T, room = 4, 3, 7, 130
    ctx = ssb.Context(B, H_kv, H_kv, d, 1, 1, 64)
    cache = make_cache(ssb, B, H_kv, d, page, room, 7 * page + d, order, pad)
    g = _gen(d + page)
    K = (torch.randn(B, H_kv, T, d, generator=g) * torch.exp2(torch.randint(-40, 30, (B, H_kv, T, 1), generator=g).float())).bfloat16()
    V = torch.randn(B, T, H_kv, d, generator=g).bfloat16().transpose(1, 2)      # strided source
    inf = float("inf")
    K[0, 0, 1] = 0.0
    K[0, 1, 1, :6] = torch.tensor([inf, -inf, float("nan"), 3.0, -1e-3, 0.0])
    K[0, 2, 1] = float("nan")
    K[1, 0, 0] = 3.38e38
    K[1, 1, 0] = 1e-39
    K[1, 2, 0, 0] = -448.0
    cnt = torch.tensor([T, 3, 0, 5], dtype=torch.int32)
    idx = torch.stack([torch.randperm(T, generator=g) for _ in range(B)]).to(torch.int32)
    idx[3, :5] = torch.tensor([2, 2, 0, 6, 6])
    off = torch.tensor([0, 127, 9, 60], dtype=torch.int32)
    before = [t.clone() for t in cache.tensors[:4]]
    ctx.ss_kv8_write(cache, K.to(DEV), V.to(DEV), off.to(DEV), cnt.to(DEV), idx.to(DEV))
    assert ctx.ss_poll_status() == (0, 0)
    want = [t.cpu().numpy().copy() for t in before]
    for b in range(B):
        for k in range(int(cnt[b])):
            (o,), (i,) = slots(cache, b, [int(off[b]) + k])
            for n, src in ((0, K), (1, V)):
                for h in range(H_kv):
                    codes, byte = kv8.encode_row(src[b, h, int(idx[b, k])].double().numpy())
                    want[n][o, h, i], want[2 + n][o, h, i] = codes, byte
    for n in (0, 1):
        got = cache.tensors[n].cpu().numpy()
        nan = (got & 0x7F == 0x7F) & (want[n] & 0x7F == 0x7F)                    # a NaN's sign is free
        assert ((got == want[n]) | nan).all()
        assert np.array_equal(cache.tensors[2 + n].cpu().numpy(), want[2 + n])
    ctx.close()


@pytest.mark.parametrize("T", [1, 2, 33, 1000])
def test_write_then_read_without_lists(T):
    """No index, count or offset: rows in order, all of them, from token 0; read back exactly."""
    ssb = _ssb()
    B, H_kv, d = 3, 2, 128
    ctx = ssb.Context(B, H_kv, H_kv, d, 1, 1, 64)
    cache = make_cache(ssb, B, H_kv, d, 16, T, T)
    g = _gen(T)
    K, V = (torch.randn(B, H_kv, T, d, generator=g).bfloat16() for _ in range(2))
    ctx.ss_kv8_write(cache, K.to(DEV), V.to(DEV))
    Kr, Vr = torch.zeros_like(K).to(DEV), torch.zeros_like(V).to(DEV)
    ctx.ss_kv8_read(cache, Kr, Vr)
    assert ctx.ss_poll_status() == (0, 0)
    for b in range(B):
        hk, hv = history(cache, b, T)
        assert np.array_equal(Kr[b].double().cpu().numpy(), hk) and np.array_equal(Vr[b].double().cpu().numpy(), hv)
        # half a step of e4m3, or of its smallest numbers at the row's scale
        top = K[b].double().abs().amax(-1, keepdim=True)
        tol = torch.maximum(2.0 ** -4 * K[b].double().abs(), top * 2.0 ** -17)   # 2^e < top / 224 * ... <= top 2^-7
        assert ((Kr[b].double().cpu() - K[b].double()).abs() <= tol).all()
    ctx.close()


def test_read_ranges_leave_other_rows_alone():
    ssb = _ssb()
    B, H_kv, d, T = 4, 2, 64, 40
    ctx = ssb.Context(B, H_kv, H_kv, d, 1, 1, 64)
    cache = make_cache(ssb, B, H_kv, d, 8, 100, 3, (0, 2, 1))
    off = torch.tensor([0, 17, 64, 99], dtype=torch.int32, device=DEV)
    cnt = torch.tensor([40, 0, 33, 1], dtype=torch.int32, device=DEV)
    K = torch.full((B, T, H_kv, d), -3.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    V = torch.full((B, H_kv, T, d), 5.0, dtype=torch.bfloat16, device=DEV)
    ctx.ss_kv8_read(cache, K, V, off, cnt)
    assert ctx.ss_poll_status() == (0, 0)
    for b in range(B):
        n, o = int(cnt[b]), int(off[b])
        hk, hv = history(cache, b, o + n)
        assert np.array_equal(K[b, :, :n].double().cpu().numpy(), hk[:, o:])
        assert np.array_equal(V[b, :, :n].double().cpu().numpy(), hv[:, o:])
        assert (K[b, :, n:] == -3.0).all() and (V[b, :, n:] == 5.0).all()
    ctx.close()


def test_device_detected_problems_are_flagged_and_skipped():
    ssb = _ssb()
    B, H_kv, d, T = 3, 1, 64, 4
    ctx = ssb.Context(B, 1, 1, d, 1, 1, 64)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    K = torch.randn(B, H_kv, T, d, device=DEV).bfloat16()

    def run(bit, cnt=None, idx=None, off=None, table=None, changed=None):
        cache = make_cache(ssb, B, H_kv, d, 8, 16, 1)
        if table is not None:
            cache.tensors[4].copy_(table(cache.tensors[4]))
        before = cache.tensors[0].clone()
        ctx.ss_kv8_write(cache, K, K, off, cnt, idx)
        st, bits = ctx.ss_poll_status()
        assert st == ssb.SS_ERR_DEVICE_FLAG and bits == bit
        assert int((cache.tensors[0] != before).any(-1).sum()) == changed

    run(ssb.SS_DEV_BAD_ACCEPT, cnt=i32(5, -1, 2), changed=4 + 0 + 2)
    run(ssb.SS_DEV_BAD_ACCEPT, idx=i32([0, 4, 1, -1], [0, 1, 2, 3], [0, 1, 2, 3]).view(B, T), changed=2 + 4 + 4)
    run(ssb.SS_DEV_DST_OVERFLOW, off=i32(14, -2, 0), changed=2 + 2 + 4)

    def broken(t):
        t = t.clone()
        t[1, 0] = 1 << 20
        return t
    run(ssb.SS_DEV_BAD_PAGE, table=broken, changed=8)

    cache = make_cache(ssb, B, H_kv, d, 8, 16, 1)
    cache.tensors[4][2, 0] = -1
    out = torch.full((B, H_kv, T, d), 9.0, dtype=torch.bfloat16, device=DEV)
    ctx.ss_kv8_read(cache, out, out.clone())
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_PAGE)
    assert (out[2] == 0).all()
    out.fill_(9.0)
    cache = make_cache(ssb, B, H_kv, d, 8, 16, 1)
    ctx.ss_kv8_read(cache, out, out.clone(), i32(13, 0, 0), i32(4, 0, 9))
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_VALID_LEN)
    assert (out[0, :, 3] == 9.0).all() and (out[1] == 9.0).all() and not (out[2] == 9.0).any()
    ctx.close()


# ------------------------------------------------------------------ attention

CASES = [
    # B, H_q, H_kv, d, T_q, lens, page, order, pad
    (1, 1, 1, 64, 1, [1], 8, (0, 1, 2), 0),
    (1, 4, 1, 128, 1, [127], 16, (0, 1, 2), 0),
    (2, 8, 2, 128, 1, [128, 129], 32, (0, 2, 1), 0),
    (3, 8, 8, 64, 1, [0, 5, 1000], 64, (0, 1, 2), 0),
    (2, 10, 2, 128, 1, [4000, 3], 128, (0, 2, 1), 16),
    (2, 16, 2, 64, 3, [700, 1531], 0, (0, 1, 2), 0),
    (4, 32, 8, 128, 1, [2000, 0, 1, 513], 256, (0, 1, 2), 0),
    (2, 8, 1, 128, 5, [300, 1111], 24, (0, 1, 2), 0),        # odd page sizes, 40 rows
    (2, 6, 2, 64, 2, [77, 400], 1, (1, 0, 2), 0),
    (2, 8, 2, 64, 4, [640, 1000], 16, (0, 1, 2), 16),
    (1, 40, 8, 128, 64, [900], 64, (0, 1, 2), 0),            # 320 rows per kv-head
    (1, 33, 1, 64, 1, [5000], 8, (0, 1, 2), 0),
    (17, 4, 2, 128, 2, [(97 * b) % 1500 for b in range(17)], 16, (0, 1, 2), 0),
    (70, 2, 1, 64, 1, [b * b % 611 for b in range(70)], 8, (0, 1, 2), 0),
]


@pytest.mark.parametrize("flags", [0, 1], ids=["auto", "simt"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}_{c[1]}x{c[2]}_d{c[3]}_T{c[4]}_p{c[6]}")
def test_attention_matches_fp64(case, flags):
    ssb = _ssb()
    B, H_q, H_kv, d, T, lens, page, order, pad = case
    room = max(max(lens), 1) + 9
    cache = make_cache(ssb, B, H_kv, d, page, room, B + d, order, pad)
    poison(cache, lens)
    Q = torch.randn(B, T, H_q, d, generator=_gen(5)).bfloat16().to(DEV).transpose(1, 2)
    ctx = ssb.Context(B, H_q, H_kv, d, T, 1, cache.desc.page_size * cache.desc.pages_per_req, flags=flags)
    O, LSE = decode(ssb, cache, Q, lens, ctx=ctx)
    if flags:
        assert ctx.last_chunk_kernel() == "kv8-simt"
    check_attention(Q, O, LSE, lambda b: history(cache, b, lens[b]), d ** -0.5)
    # again, bit for bit (the join does not depend on which CTA comes last)
    O2, LSE2 = decode(ssb, cache, Q, lens, ctx=ctx)
    assert torch.equal(O.view(torch.int16), O2.view(torch.int16)) and torch.equal(LSE, LSE2)
    ctx.close()


@pytest.mark.parametrize("kind", ["peaked", "sink", "falling", "rising", "wide_v", "wide_k", "wide_q", "equal"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_uneven_values(kind, d):
    """Weights spread over many binades, tokens and heads of very different magnitude."""
    ssb = _ssb()
    B, H_q, H_kv, n = 1, 8, 2, 6000
    cache = make_cache(ssb, B, H_kv, d, 64, n, 11)
    g = _gen(3)
    K, V = torch.randn(B, H_kv, n, d, generator=g), torch.randn(B, H_kv, n, d, generator=g)
    Q = torch.randn(B, H_q, 1, d, generator=g)
    u = torch.sign(torch.randn(d, generator=g))
    t = torch.arange(n).view(1, 1, n, 1) / n
    if kind == "peaked":
        K = K * 8
    elif kind == "sink":                     # one token outweighs the 6000 others together, its V is small
        K, Q = K * 0.1, Q * 0.1 + u * 0.3
        K[:, :, 0], V[:, :, 0] = 4 * u, V[:, :, 0] * 2.0 ** -6
    elif kind == "falling":                  # the first tile's maximum is far above every later one
        K, Q = K * 0.1 + u * (1 - t) * 4, Q * 0.1 + u * 0.3
    elif kind == "rising":
        K, Q = K * 0.1 + u * t * 4, Q * 0.1 + u * 0.3
    elif kind == "wide_v":
        V = V * torch.exp2(torch.randint(-24, 60, (1, 1, n, 1), generator=g).float())
    elif kind == "wide_k":
        K = K * torch.exp2(torch.randint(-30, 2, (1, 1, n, 1), generator=g).float())
    elif kind == "wide_q":
        Q = Q * torch.exp2(torch.arange(H_q).view(1, H_q, 1, 1) * 1.5 - 8)
        Q[..., ::7] *= 2.0 ** -9
    else:
        K = K[:, :, :1].expand_as(K)
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, cache.desc.page_size * cache.desc.pages_per_req)
    ctx.ss_kv8_write(cache, K.bfloat16().contiguous().to(DEV), V.bfloat16().to(DEV))
    Q = Q.bfloat16().to(DEV)
    O, LSE = decode(ssb, cache, Q, [n], ctx=ctx)
    check_attention(Q, O, LSE, lambda b: history(cache, b, n), d ** -0.5)
    ctx.close()


def test_no_lengths_means_the_whole_room_and_all_empty_batches():
    ssb = _ssb()
    cache = make_cache(ssb, 2, 2, 128, 16, 200, 5)
    Q = torch.randn(2, 4, 1, 128, generator=_gen(1)).bfloat16().to(DEV)
    O, LSE = decode(ssb, cache, Q, None)
    check_attention(Q, O, LSE, lambda b: history(cache, b, 208), 128 ** -0.5)
    O, LSE = decode(ssb, cache, Q, [0, 0])
    assert (O == 0).all() and (LSE == -math.inf).all()


def test_bad_lengths_and_pages_are_flagged():
    ssb = _ssb()
    B, d, page = 3, 128, 16
    cache = make_cache(ssb, B, 2, d, page, 300, 6)
    room = page * cache.desc.pages_per_req
    Q = torch.randn(B, 4, 1, d, generator=_gen(1)).bfloat16().to(DEV)
    ctx = ssb.Context(B, 4, 2, d, 1, 1, room)
    O, LSE = torch.empty_like(Q), torch.empty(B, 4, 1, device=DEV)
    vl = torch.tensor([room + 1, -1, 40], dtype=torch.int32, device=DEV)
    ctx.ss_decode8(Q, 0.1, cache, vl, O, LSE)
    assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_VALID_LEN)
    check_attention(Q, O, LSE, lambda b: history(cache, b, [room, 0, 40][b]), 0.1)
    # a page outside the pool reads as zeros: scores 0, values 0
    K, V, Ks, Vs, table = cache.tensors
    o, i = slots(cache, 1, np.arange(32, 48))
    ref = [history(cache, b, 100) for b in range(B)]
    for bad in (-1, K.shape[0], 2 ** 31 - 1):
        table[1, 2] = bad
        ref[1][0][:, 32:48] = 0
        ref[1][1][:, 32:48] = 0
        ctx.ss_decode8(Q, 0.1, cache, torch.full((B,), 100, dtype=torch.int32, device=DEV), O, LSE)
        assert ctx.ss_poll_status() == (ssb.SS_ERR_DEVICE_FLAG, ssb.SS_DEV_BAD_PAGE)
        check_attention(Q, O, LSE, lambda b: ref[b], 0.1)
    ctx.close()


def test_refusals():
    ssb = _ssb()
    B, H_kv, d = 2, 2, 64
    ctx = ssb.Context(B, 4, H_kv, d, 2, 2, 256)
    lib, h = ctx.lib, ctx.handle
    cache = make_cache(ssb, B, H_kv, d, 16, 256, 1)
    Q = torch.randn(B, 4, 1, d, device=DEV).bfloat16()
    O, L = torch.empty_like(Q), torch.empty(B, 4, 1, device=DEV)
    x = torch.randn(B, H_kv, 4, d, device=DEV).bfloat16()
    launches = ctx.launch_count()

    def desc(**kw):
        c = ssb.ss_cache8()
        C.memmove(C.byref(c), C.byref(cache.desc), C.sizeof(c))
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    def t8(t, **kw):
        r = ssb.ss_tensor(t.ptr, t.stride_b, t.stride_h, t.stride_t)
        for k, v in kw.items():
            setattr(r, k, v)
        return r

    k = cache.desc.K
    bad = [(ssb.SS_ERR_ARG, desc(K=t8(k, ptr=None))), (ssb.SS_ERR_ARG, desc(V_scale=t8(k, ptr=None))),
           (ssb.SS_ERR_ARG, desc(n_pages=0)), (ssb.SS_ERR_ARG, desc(page_size=0)), (ssb.SS_ERR_ARG, desc(pages_per_req=0)),
           (ssb.SS_ERR_SHAPE, desc(page_table=None, n_pages=1)), (ssb.SS_ERR_SHAPE, desc(page_size=1 << 16, pages_per_req=1 << 15)),
           (ssb.SS_ERR_ALIGN, desc(K=t8(k, ptr=k.ptr + 8))), (ssb.SS_ERR_ALIGN, desc(V=t8(k, stride_t=72))),
           (ssb.SS_ERR_ALIGN, desc(page_table=cache.desc.page_table + 2))]
    qt, xt = ssb.as_ss_tensor(Q), ssb.as_ss_tensor(x)
    s = ctx._sp(None)
    dec = lambda c, q=qt, B=B, T=1, scale=1.0, o=O.data_ptr(), l=L.data_ptr(), vl=None: lib.ss_decode8(
        h, q, B, T, scale, C.byref(c), vl, o, l, s)
    wr = lambda c, a=xt, B=B, T=4, i=None, n=None, o=None: lib.ss_kv8_write(h, C.byref(c), a, a, B, T, i, n, o, s)
    rd = lambda c, a=xt, B=B, T=4, n=None, o=None: lib.ss_kv8_read(h, C.byref(c), a, a, B, T, o, n, s)
    for want, c in bad:
        assert dec(c) == want and wr(c) == want and rd(c) == want, want
    good = desc()
    assert dec(desc(pages_per_req=17)) == ssb.SS_ERR_SHAPE                        # more room than max_Lc
    assert dec(good, B=3) == ssb.SS_ERR_SHAPE and dec(good, T=3) == ssb.SS_ERR_SHAPE
    assert dec(good, B=0) == ssb.SS_ERR_ARG and dec(good, T=0) == ssb.SS_ERR_ARG
    assert dec(good, scale=0.0) == ssb.SS_ERR_ARG and dec(good, scale=float("nan")) == ssb.SS_ERR_ARG
    assert dec(good, o=None) == ssb.SS_ERR_ARG and dec(good, o=O.data_ptr() + 2) == ssb.SS_ERR_ALIGN
    assert dec(good, l=L.data_ptr() + 2) == ssb.SS_ERR_ALIGN and dec(good, vl=L.data_ptr() + 2) == ssb.SS_ERR_ALIGN
    assert dec(good, q=t8(qt, stride_h=12)) == ssb.SS_ERR_ALIGN
    for f in (wr, rd):
        assert f(good, B=3) == ssb.SS_ERR_SHAPE and f(good, T=1 << 29) == ssb.SS_ERR_SHAPE
        assert f(good, T=0) == ssb.SS_ERR_ARG and f(good, a=t8(xt, ptr=None)) == ssb.SS_ERR_ARG
        assert f(good, a=t8(xt, stride_t=4)) == ssb.SS_ERR_ALIGN and f(good, n=L.data_ptr() + 1) == ssb.SS_ERR_ALIGN
    # order of calls
    assert lib.ss_verify_chunk8(h, C.byref(good), None, s) == ssb.SS_ERR_STATE
    ctx.ss_verify_begin(Q, 1.0)
    assert dec(good) == ssb.SS_ERR_STATE
    for want, c in bad + [(ssb.SS_ERR_SHAPE, desc(pages_per_req=17))]:
        assert lib.ss_verify_chunk8(h, C.byref(c), None, s) == want
    ctx.ss_verify_abort()
    assert ctx.launch_count() == launches
    ctx.close()


def test_round_of_bf16_and_8_bit_chunks():
    """History in three pieces (8 bits paged, bf16, 8 bits dense) and the local segment against one fp64 softmax."""
    ssb = _ssb()
    B, H_q, H_kv, d, T = 3, 8, 2, 128, 5
    lens = [[300, 0, 77], [64, 128, 1], [0, 511, 40]]                  # piece, request
    A, Z = make_cache(ssb, B, H_kv, d, 16, 320, 1), make_cache(ssb, B, H_kv, d, 0, 520, 2)
    g = _gen(9)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)
    K, V, Kl, Vl, Q = rnd(B, H_kv, 128, d), rnd(B, H_kv, 128, d), rnd(B, H_kv, T, d), rnd(B, H_kv, T, d), rnd(B, H_q, T, d)
    poison(A, lens[0])
    poison(Z, lens[2])
    vls = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in lens]
    for overlap in (0, ssb.SS_FLAG_OVERLAP_CHUNKS):
        for order in ((0, 1, 2), (2, 1, 0), (1, 0, 2)):
            ctx = ssb.Context(B, H_q, H_kv, d, T, T, 1024, max_chunks=2, flags=overlap)
            O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
            for _ in range(3):                                         # the same context, round after round
                O.zero_(), LSE.zero_()
                ctx.ss_verify_begin(Q, d ** -0.5)
                for x in order:
                    if x == 0: ctx.ss_verify_chunk8(A, vls[0])
                    elif x == 1: ctx.ss_verify_chunk(K, V, vls[1])
                    else: ctx.ss_verify_chunk8(Z, vls[2])
                ctx.ss_verify_local(Kl, Vl)
                ctx.ss_verify_finalize(O, LSE)
                assert ctx.ss_poll_status() == (0, 0)
            # every candidate row sees a different local segment: one fp64 softmax per row
            for i in range(T):
                def kv(b):
                    a, z = history(A, b, lens[0][b]), history(Z, b, lens[2][b])
                    f = lambda t, n: t[b, :, :n].double().cpu().numpy()
                    return (np.concatenate([a[0], f(K, lens[1][b]), z[0], f(Kl, i + 1)], 1),
                            np.concatenate([a[1], f(V, lens[1][b]), z[1], f(Vl, i + 1)], 1))
                check_attention(Q[:, :, i:i + 1], O[:, :, i:i + 1], LSE[:, :, i:i + 1], kv, d ** -0.5)
            ctx.close()


def test_captured_decode_follows_lengths_and_pages():
    """One captured step (write the new token, attend) replayed while the requests grow and empty ones join."""
    ssb = _ssb()
    B, H_q, H_kv, d, page = 3, 8, 2, 128, 16
    cache = make_cache(ssb, B, H_kv, d, page, 2000, 8)
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 2048, flags=ssb.SS_FLAG_OVERLAP_CHUNKS)
    g = _gen(2)
    K, V = (torch.zeros(B, H_kv, 1, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    Q = torch.zeros(B, H_q, 1, d, dtype=torch.bfloat16, device=DEV)
    O, LSE = torch.empty_like(Q), torch.empty(B, H_q, 1, device=DEV)
    off = torch.zeros(B, dtype=torch.int32, device=DEV)
    n = torch.zeros(B, dtype=torch.int32, device=DEV)

    def step():
        ctx.ss_kv8_write(cache, K, V, off)
        ctx.ss_decode8(Q, d ** -0.5, cache, n, O, LSE)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([1, 1, 1], [1500, 2, 1999], [64, 700, 128], [0, 1, 129], [1024, 1025, 1023]):
        for t in (K, V, Q):
            t.copy_(torch.randn(t.shape, generator=g).bfloat16())
        off.copy_(torch.tensor([max(0, x - 1) for x in lens], dtype=torch.int32))
        n.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.ss_poll_status() == (0, 0)
        check_attention(Q, O, LSE, lambda b: history(cache, b, lens[b]), d ** -0.5)
        got = O.clone(), LSE.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0].view(torch.int16), O.view(torch.int16)) and torch.equal(got[1], LSE)
    ctx.close()


def test_streams_and_contexts_side_by_side():
    """Two contexts on two streams at once, neither the current one."""
    ssb = _ssb()
    runs = []
    for k in range(2):
        cache = make_cache(ssb, 2, 2, 128, 32, 3000, 20 + k)
        Q = torch.randn(2, 8, 1, 128, generator=_gen(k)).bfloat16().to(DEV)
        O, LSE = torch.empty_like(Q), torch.empty(2, 8, 1, device=DEV)
        ctx = ssb.Context(2, 8, 2, 128, 1, 1, 4096)
        runs.append((ctx, cache, Q, torch.tensor([3000, 17 + k], dtype=torch.int32, device=DEV), O, LSE, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for ctx, cache, Q, n, O, LSE, st in runs:
            ctx.ss_decode8(Q, 0.09, cache, n, O, LSE, stream=st)
    torch.cuda.synchronize()
    for k, (ctx, cache, Q, n, O, LSE, st) in enumerate(runs):
        check_attention(Q, O, LSE, lambda b: history(cache, b, [3000, 17 + k][b]), 0.09)
        ctx.close()


@pytest.mark.parametrize("page", [0, 64])
def test_offsets_past_32_bits(page):
    """Codes more than 2^32 bytes into the cache: written, read back and attended to."""
    ssb = _ssb()
    H_kv, d, tokens, n = 2, 128, 300, 300
    if page:
        outer = (1 << 32) // (H_kv * page * d) + 70
        shape = (outer, H_kv, page, d)
        table = torch.arange(outer - 8, outer, dtype=torch.int32, device=DEV).view(1, 8)[:, :5].contiguous()
        B = 1
    else:
        shape, table, B = (2, H_kv, 320, d), None, 2
    if page:
        K, V = (torch.empty(shape, dtype=torch.uint8, device=DEV) for _ in range(2))
    else:                                                             # two requests 4 GiB and a bit apart
        K, V = (torch.empty((1 << 32) + (1 << 20), dtype=torch.uint8, device=DEV).as_strided(
            shape, ((1 << 32) + 4096, 320 * d, d, 1)) for _ in range(2))
    Ks, Vs = (torch.empty(shape[:3], dtype=torch.uint8, device=DEV) for _ in range(2))
    cache = ssb.Cache8(K, V, Ks, Vs, table)
    ctx = ssb.Context(B, 4, H_kv, d, 1, 1, 512)
    g = _gen(4)
    x, y = (torch.randn(B, H_kv, n, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    ctx.ss_kv8_write(cache, x, y)
    xr, yr = torch.zeros_like(x), torch.zeros_like(y)
    ctx.ss_kv8_read(cache, xr, yr)
    Q = torch.randn(B, 4, 1, d, generator=g).bfloat16().to(DEV)
    O, LSE = decode(ssb, cache, Q, [n] * B, ctx=ctx)
    enc = lambda t, b: np.stack([kv8.decode(*kv8.encode_row(r)) for r in t[b].double().cpu().numpy().reshape(-1, d)]).reshape(H_kv, n, d)
    for b in range(B):
        assert np.array_equal(xr[b].double().cpu().numpy(), enc(x, b)) and np.array_equal(yr[b].double().cpu().numpy(), enc(y, b))
    check_attention(Q, O, LSE, lambda b: (enc(x, b), enc(y, b)), d ** -0.5)
    ctx.close()


def test_a_generation_as_it_would_run():
    """Prompts written, then steps of: accepted rows written, decode; at the end the histories read back."""
    ssb = _ssb()
    B, H_q, H_kv, d, page, steps = 3, 16, 4, 64, 16, 6
    g = _gen(31)
    prompt = [130, 1, 47]
    room = 256
    cache = make_cache(ssb, B, H_kv, d, page, room, 13)
    ctx = ssb.Context(B, H_q, H_kv, d, 4, 4, room)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    want = [[np.zeros((H_kv, 0, d))] * 2 for _ in range(B)]

    def add(b, K, V, rows):
        for k, t in ((0, K), (1, V)):
            new = np.stack([np.stack([kv8.decode(*kv8.encode_row(t[b, h, r].double().cpu().numpy())) for r in rows])
                            if len(rows) else np.zeros((0, d)) for h in range(H_kv)])
            want[b][k] = np.concatenate([want[b][k], new], 1)
    K, V = rnd(B, H_kv, max(prompt), d), rnd(B, H_kv, max(prompt), d)
    ctx.ss_kv8_write(cache, K, V, None, i32(prompt))
    lens = list(prompt)
    for b in range(B):
        add(b, K, V, range(prompt[b]))
    for step in range(steps):
        T = 4
        K, V, Q = rnd(B, H_kv, T, d), rnd(B, H_kv, T, d), rnd(B, H_q, 1, d)
        acc = [(step + b) % 4 + 1 for b in range(B)]
        idx = torch.stack([torch.randperm(T, generator=g).sort().values for _ in range(B)]).to(torch.int32).to(DEV)
        ctx.ss_kv8_write(cache, K, V, i32(lens), i32(acc), idx)
        for b in range(B):
            add(b, K, V, range(acc[b]))
            lens[b] += acc[b]
        O, LSE = decode(ssb, cache, Q, lens, ctx=ctx)
        check_attention(Q, O, LSE, lambda b: want[b], d ** -0.5)
    Kr, Vr = torch.zeros(B, H_kv, room, d, dtype=torch.bfloat16, device=DEV), torch.zeros(B, H_kv, room, d, dtype=torch.bfloat16, device=DEV)
    ctx.ss_kv8_read(cache, Kr, Vr, None, i32(lens))
    for b in range(B):
        assert np.array_equal(Kr[b, :, :lens[b]].double().cpu().numpy(), want[b][0])
        assert np.array_equal(Vr[b, :, :lens[b]].double().cpu().numpy(), want[b][1])
        assert (Kr[b, :, lens[b]:] == 0).all()
    ctx.close()


@pytest.mark.parametrize("page,kernel", [(0, "kv8-tcgen05"), (8, "kv8-tcgen05"), (64, "kv8-tcgen05"), (256, "kv8-tcgen05"),
                                         (4, "kv8-simt"), (24, "kv8-simt"), (192, "kv8-simt")])
def test_which_kernel_runs(page, kernel):
    ssb = _ssb()
    cache = make_cache(ssb, 1, 2, 64, page, 500, 1)
    Q = torch.randn(1, 4, 1, 64, generator=_gen(1)).bfloat16().to(DEV)
    ctx = ssb.Context(1, 4, 2, 64, 1, 1, 1024)
    O, LSE = decode(ssb, cache, Q, [500], ctx=ctx)
    assert ctx.last_chunk_kernel() == kernel
    check_attention(Q, O, LSE, lambda b: history(cache, b, 500), 64 ** -0.5)
    ctx.close()


MORE = [
    # B, H_q, H_kv, d, T_q, lens, page, order, pad
    (2, 8, 2, 128, 3, [5000, 131], 64, (0, 1, 2), 0),                    # 12 rows
    (2, 16, 2, 128, 4, [2600, 999], 16, (0, 2, 1), 0),                   # 32 rows
    (2, 10, 2, 128, 8, [1300, 700], 8, (0, 1, 2), 16),                   # 40 rows in two tiles
    (1, 8, 1, 128, 1, [40001], 128, (0, 1, 2), 0),                       # more CTAs than 128-token pages per share
    (1, 16, 1, 64, 2, [70000], 64, (0, 1, 2), 0),
    (3, 6, 3, 128, 1, [1152, 700, 384], 384, (0, 1, 2), 0),              # pages of three tiles
    (2, 4, 2, 64, 1, [1025, 1024], 0, (0, 2, 1), 16),                    # dense, tokens interleaved with heads
    (40, 4, 4, 128, 1, [1 + (b * 53) % 300 for b in range(40)], 32, (0, 1, 2), 0),
    (33, 5, 1, 64, 7, [0 if b % 3 else 200 + b for b in range(33)], 16, (0, 1, 2), 0),
]


@pytest.mark.parametrize("case", MORE, ids=lambda c: f"B{c[0]}_{c[1]}x{c[2]}_d{c[3]}_T{c[4]}_p{c[6]}")
def test_attention_on_the_tensor_cores(case):
    ssb = _ssb()
    B, H_q, H_kv, d, T, lens, page, order, pad = case
    cache = make_cache(ssb, B, H_kv, d, page, max(lens) + 30, B + d, order, pad)
    poison(cache, lens)
    Q = torch.randn(B, H_q, T, d, generator=_gen(6)).bfloat16().to(DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, T, 1, cache.desc.page_size * cache.desc.pages_per_req)
    O, LSE = decode(ssb, cache, Q, lens, ctx=ctx)
    assert ctx.last_chunk_kernel() == "kv8-tcgen05"
    check_attention(Q, O, LSE, lambda b: history(cache, b, lens[b]), d ** -0.5)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ctx.ss_decode8(Q, d ** -0.5, cache, vl, O.zero_(), None)             # LSE is optional
    again, _ = decode(ssb, cache, Q, lens, ctx=ctx)
    assert torch.equal(O.view(torch.int16), again.view(torch.int16))
    ctx.close()


def test_calls_back_to_back_on_one_context():
    """Large and small batches (units cut and whole, with and without a join) in one stream without a wait between
    them: every result as when it is computed alone."""
    ssb = _ssb()
    H_q, H_kv, d = 8, 2, 128
    ctx = ssb.Context(6, H_q, H_kv, d, 4, 4, 8192, flags=ssb.SS_FLAG_OVERLAP_CHUNKS)
    jobs = []
    for k, (B, T, page, lens) in enumerate([(1, 1, 64, [8000]), (6, 1, 16, [3, 90, 128, 1, 17, 60]), (2, 4, 64, [5000, 1]),
                                            (1, 1, 128, [100]), (6, 3, 32, [700] * 6), (3, 1, 0, [0, 0, 129])]):
        cache = make_cache(ssb, B, H_kv, d, page, max(lens) + 1, 40 + k)
        Q = torch.randn(B, H_q, T, d, generator=_gen(k)).bfloat16().to(DEV)
        vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
        alone = decode(ssb, cache, Q, lens, ctx=ctx)
        check_attention(Q, *alone, lambda b: history(cache, b, lens[b]), d ** -0.5)
        jobs.append((cache, Q, vl, alone))
    outs = []
    for turn in range(5):
        for k in np.random.RandomState(turn).permutation(len(jobs)):
            cache, Q, vl, alone = jobs[k]
            O, LSE = torch.empty_like(alone[0]), torch.empty_like(alone[1])
            ctx.ss_decode8(Q, d ** -0.5, cache, vl, O, LSE)
            outs.append((k, O, LSE))
    torch.cuda.synchronize()
    assert ctx.ss_poll_status() == (0, 0)
    for k, O, LSE in outs:
        assert torch.equal(O.view(torch.int16), jobs[k][3][0].view(torch.int16)) and torch.equal(LSE, jobs[k][3][1]), k
    ctx.close()


def test_a_query_that_is_not_finite_spoils_its_own_row_only():
    ssb = _ssb()
    H_q, H_kv, d, n = 8, 2, 128, 500
    cache = make_cache(ssb, 1, H_kv, d, 16, n, 3)
    Q = torch.randn(1, H_q, 2, d, generator=_gen(1)).bfloat16().to(DEV)
    bad = Q.clone()
    bad[0, 1, 0, 7], bad[0, 6, 1, 100] = float("nan"), float("inf")
    good, gl = decode(ssb, cache, Q, [n])
    O, LSE = decode(ssb, cache, bad, [n])
    hit = torch.zeros(1, H_q, 2, dtype=torch.bool, device=DEV)
    hit[0, 1, 0] = hit[0, 6, 1] = True
    assert torch.isnan(O[hit]).all() and torch.isnan(LSE[hit]).all()
    assert torch.equal(O[~hit], good[~hit]) and torch.equal(LSE[~hit], gl[~hit])


def test_state_of_an_8_bit_chunk_can_be_exported():
    """The chunk's merged state leaves one round and enters another as any partial state does."""
    ssb = _ssb()
    B, H_q, H_kv, d, T = 2, 8, 2, 128, 3
    lens = [900, 140]
    cache = make_cache(ssb, B, H_kv, d, 64, 1000, 4)
    poison(cache, lens)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    Q = torch.randn(B, H_q, T, d, generator=_gen(2)).bfloat16().to(DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, T, T, 1024)
    rows = B * H_q * T
    ml, a = torch.empty(rows, 2, device=DEV), torch.empty(rows, d, device=DEV)
    O, LSE = torch.empty_like(Q), torch.empty(B, H_q, T, device=DEV)
    ctx.ss_verify_begin(Q, 0.1)
    ctx.ss_verify_chunk8(cache, vl)
    ctx.ss_verify_export_state(ml, a)
    ctx.ss_verify_abort()
    ctx.ss_verify_begin(Q, 0.1)
    ctx.ss_verify_import_state(ml, a)
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (0, 0)
    check_attention(Q, O, LSE, lambda b: history(cache, b, lens[b]), 0.1)
    ctx.close()


@pytest.mark.parametrize("T", [64, 65, 130, 700])
def test_writes_across_block_sizes(T):
    """Rows that end inside a block of either size, small and large calls, counts and offsets of their own."""
    ssb = _ssb()
    for B, H_kv, d in ((3, 2, 64), (24, 8, 128)):
        ctx = ssb.Context(B, H_kv, H_kv, d, 1, 1, 64)
        cache = make_cache(ssb, B, H_kv, d, 16, T + 40, T + B)
        g = _gen(T)
        K, V = (torch.randn(B, H_kv, T, d, generator=g).bfloat16() for _ in range(2))
        cnt = torch.tensor([(T * (b + 1)) // B for b in range(B)], dtype=torch.int32, device=DEV)
        off = torch.tensor([(7 * b) % 41 for b in range(B)], dtype=torch.int32, device=DEV)
        ctx.ss_kv8_write(cache, K.to(DEV), V.to(DEV), off, cnt)
        Kr, Vr = (torch.full((B, H_kv, T, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ctx.ss_kv8_read(cache, Kr, Vr, off, cnt)
        assert ctx.ss_poll_status() == (0, 0)
        for b in range(0, B, 5):
            n = int(cnt[b])
            for src, got in ((K, Kr), (V, Vr)):
                for h in range(H_kv):
                    for r in {0, n // 2, n - 1}:
                        want = kv8.decode(*kv8.encode_row(src[b, h, r].double().numpy()))
                        assert np.array_equal(got[b, h, r].double().cpu().numpy(), want), (b, h, r)
                assert (got[b, :, n:] == 3.0).all()
        ctx.close()


@pytest.mark.parametrize("B", [128, 131, 300])
def test_large_batches(B):
    """More requests than a warp looks up in one step, most of them empty or short; whole rounds too."""
    ssb = _ssb()
    H_q, H_kv, d, page = 4, 1, 64, 16
    lens = [(0 if b % 5 == 2 else (b * 37) % 400 if b % 7 else 0) for b in range(B)]
    cache = make_cache(ssb, B, H_kv, d, page, 416, B)
    poison(cache, lens)
    Q = torch.randn(B, H_q, 2, d, generator=_gen(B)).bfloat16().to(DEV)
    ctx = ssb.Context(B, H_q, H_kv, d, 2, 2, 512)
    O, LSE = decode(ssb, cache, Q, lens, ctx=ctx)
    check_attention(Q, O, LSE, lambda b: history(cache, b, lens[b]), d ** -0.5)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    O2, LSE2 = torch.empty_like(O), torch.empty_like(LSE)
    ctx.ss_verify_begin(Q, d ** -0.5)
    ctx.ss_verify_chunk8(cache, vl)
    vl.fill_(1)                                    # the round keeps to the lengths that the chunk went by
    ctx.ss_verify_finalize(O2, LSE2)
    assert ctx.ss_poll_status() == (0, 0)
    check_attention(Q, O2, LSE2, lambda b: history(cache, b, lens[b]), d ** -0.5)
    ctx.close()


def test_tensors_on_another_device_are_refused():
    ssb = _ssb()
    B, H_kv, d = 2, 2, 64
    ctx = ssb.Context(B, 4, H_kv, d, 2, 2, 64)
    cache, there = ssb.Cache8.empty(B, H_kv, 64, d), ssb.Cache8.empty(B, H_kv, 64, d, device="cpu")
    Q, x = torch.zeros(B, 4, 1, d, dtype=torch.bfloat16, device=DEV), torch.zeros(B, H_kv, 2, d, dtype=torch.bfloat16, device=DEV)
    O, L, n = torch.empty_like(Q), torch.empty(B, 4, 1, device=DEV), torch.ones(B, dtype=torch.int32, device=DEV)
    launches = ctx.launch_count()
    for args in ((there, x, x), (cache, x.cpu(), x), (cache, x, x.cpu())):
        for f in (ctx.ss_kv8_write, ctx.ss_kv8_read):
            with pytest.raises(AssertionError):
                f(*args)
    for f in (ctx.ss_kv8_write, ctx.ss_kv8_read):
        with pytest.raises(AssertionError):
            f(cache, x, x, row_cnt=n.cpu())
    for args in ((Q.cpu(), 1.0, cache, n, O, L), (Q, 1.0, there, n, O, L), (Q, 1.0, cache, n.cpu(), O, L),
                 (Q, 1.0, cache, n, O.cpu(), L), (Q, 1.0, cache, n, O, L.cpu())):
        with pytest.raises(AssertionError):
            ctx.ss_decode8(*args)
    with pytest.raises(AssertionError):
        ssb.Cache8(cache.tensors[0], *there.tensors[1:4])
    assert ctx.launch_count() == launches
    ctx.close()


def test_rows_and_pages_given_twice():
    """A row may be a source several times, and requests may share pages that they only read."""
    ssb = _ssb()
    B, H_q, H_kv, d, page = 2, 4, 2, 128, 16
    cache = ssb.Cache8.empty(8, H_kv, page, d, torch.tensor([[5, 2, 5, 7], [5, 2, 0, 1]], dtype=torch.int32, device=DEV))
    ctx = ssb.Context(B, H_q, H_kv, d, 1, 1, 4 * page)
    g = torch.Generator().manual_seed(3)
    K, V = (torch.randn(B, H_kv, 4, d, generator=g).bfloat16().to(DEV) for _ in range(2))
    idx = torch.tensor([[2, 2, 0, 2], [1, 1, 1, 1]], dtype=torch.int32, device=DEV)
    off = torch.tensor([48, 40], dtype=torch.int32, device=DEV)     # pages 7 and 0
    ctx.ss_kv8_write(cache, K, V, dst_off=off, row_idx=idx)
    Kr, Vr = torch.empty_like(K), torch.empty_like(V)
    ctx.ss_kv8_read(cache, Kr, Vr, src_off=off)
    for b in range(B):
        for k in range(4):
            src = int(idx[b, k])
            first = idx[b].tolist().index(src)
            for got, rows in ((Kr, K), (Vr, V)):
                assert torch.equal(got[b, :, k], got[b, :, first])
                want = rows[b, :, src].double()
                top = want.abs().amax(-1, keepdim=True)
                # half a step of e4m3: 2^-4 of the value, or 2^-10 * 2^e with 2^e < 2 * top / 448
                tol = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -9 / 448 * top)
                assert ((got[b, :, k].double() - want).abs() <= tol).all()
    # page 5 twice in one request and in both
    fill = torch.randn(1, H_kv, 32, d, generator=g).bfloat16().to(DEV)
    ctx.ss_kv8_write(ssb.Cache8(*cache.tensors[:4], cache.tensors[4][:1].contiguous()), fill, fill)
    Kr, Vr = (torch.empty(B, H_kv, 48, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.ss_kv8_read(cache, Kr, Vr)
    assert torch.equal(Kr[0, :, :16], Kr[0, :, 32:]) and torch.equal(Kr[0, :, :32], Kr[1, :, :32])
    Q = torch.randn(B, H_q, 1, d, generator=g).bfloat16().to(DEV)
    O, L = torch.empty_like(Q), torch.empty(B, H_q, 1, device=DEV)
    n = torch.tensor([48, 32], dtype=torch.int32, device=DEV)
    ctx.ss_decode8(Q, d ** -0.5, cache, n, O, L)
    for b in range(B):
        for h in range(H_q):
            rows = int(n[b])
            k, v = (t[b, h // 2, :rows].double().cpu().numpy() for t in (Kr, Vr))
            o, lse, A = kv8.attention(Q[b, h].double().cpu().numpy(), k, v, d ** -0.5)
            err = np.abs(O[b, h].double().cpu().numpy() - o)
            # bf16 output (2^-8 of the value) and weights of 9 bits (2^-9 of the sum of |w v|)
            assert (err <= 2.0 ** -8 * np.abs(o) + 2.0 ** -8 * A).all()
            assert abs(float(L[b, h, 0]) - lse[0]) < 1e-4
    assert ctx.ss_poll_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("rows", [12, 17, 24, 25, 32, 40, 48, 51])
@pytest.mark.parametrize("kind", ["rising", "sink", "wide_v"])
@pytest.mark.parametrize("d", [64, 128])
def test_uneven_values_with_many_rows(rows, kind, d):
    """References raised in mid-stream, and scales far apart, for every number of rows per tile; a row's
    scores grow at its own pace."""
    ssb = _ssb()
    B, H_kv, lens = 2, 2, [2900, 140]
    n = max(lens)
    cache = make_cache(ssb, B, H_kv, d, 32, n, 17)
    g = _gen(rows)
    K, V = torch.randn(B, H_kv, n, d, generator=g), torch.randn(B, H_kv, n, d, generator=g)
    Q = torch.randn(B, H_kv * rows, 1, d, generator=g)
    u = torch.sign(torch.randn(d, generator=g))
    t = torch.arange(n).view(1, 1, n, 1) / n
    pace = (torch.arange(H_kv * rows) % rows + 1).view(1, -1, 1, 1) / rows
    if kind == "rising":
        K, Q = K * 0.1 + u * t * 4, Q * 0.1 + u * 0.3 * pace
    elif kind == "sink":
        K, Q = K * 0.1, Q * 0.1 + u * 0.3 * pace
        K[:, :, 0], V[:, :, 0] = 4 * u, V[:, :, 0] * 2.0 ** -6
    else:
        V = V * torch.exp2(torch.randint(-24, 60, (1, 1, n, 1), generator=g).float())
    ctx = ssb.Context(B, H_kv * rows, H_kv, d, 1, 1, cache.desc.page_size * cache.desc.pages_per_req)
    ctx.ss_kv8_write(cache, K.bfloat16().to(DEV), V.bfloat16().to(DEV))
    Q = Q.bfloat16().to(DEV)
    O, LSE = decode(ssb, cache, Q, lens, ctx=ctx)
    assert ctx.last_chunk_kernel() == "kv8-tcgen05"
    check_attention(Q, O, LSE, lambda b: history(cache, b, lens[b]), d ** -0.5)
    ctx.close()
