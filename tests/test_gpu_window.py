"""Attention over a window with sinks on the GPU, over bf16 and 8-bit caches, against its definition in fp64."""
import numpy as np
import pytest
import torch

from oracle import kv8
from tests import test_gpu_kv8 as t8
from tests.test_gpu_rope import _cache16, _slots16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ssb():
    from paper_2609_33184_b200 import binding
    return binding


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def make(ssb, bits, B, H_kv, d, page, room, seed, order=(0, 1, 2)):
    return t8.make_cache(ssb, B, H_kv, d, page, room, seed, order) if bits == 8 else _cache16(ssb, B, H_kv, d, page, room, seed, order)


def places(cache, b, tokens):
    return t8.slots(cache, b, tokens) if len(cache.tensors) == 5 else _slots16(cache, b, tokens)


def history(cache, b, tokens):
    """fp64 K, V [H_kv, n, d] of some of request b's tokens."""
    o, i = places(cache, b, tokens)
    out = []
    for k in (0, 1):
        x = cache.tensors[k][torch.as_tensor(o, device=DEV), :, torch.as_tensor(i, device=DEV)].cpu()
        if len(cache.tensors) == 5:
            byte = cache.tensors[2 + k][torch.as_tensor(o, device=DEV), :, torch.as_tensor(i, device=DEV)].cpu().numpy()
            x = kv8.decode(x.numpy(), byte)
        else:
            x = x.double().numpy()
        out.append(x.transpose(1, 0, 2))
    return out


def seen_by(p, n, window, sinks):
    """Tokens that a query at position p sees of a request of n tokens."""
    j = np.arange(n)
    return j[(j <= p) & ((j < sinks) | (p - j < window))]


def positions(n, T, depth=None, decode=True):
    return [n - T + t for t in range(T)] if decode else [n + (t if depth is None else depth[t]) for t in range(T)]


def hide(cache, lens, T, window, sinks, room, depth=None, decode=True):
    """What no query sees becomes NaN (8 bits: NaN codes, scale bytes 255), the ids of pages without a seen token wrong."""
    table = cache.tensors[-1]
    page = cache.tensors[0].shape[2]
    for b, n in enumerate(lens):
        seen = np.zeros(room, dtype=bool)
        for p in positions(n, T, None if depth is None else depth[b], decode):
            seen[seen_by(p, n, window, sinks)] = True
        o, i = (torch.as_tensor(x, device=DEV) for x in places(cache, b, np.nonzero(~seen)[0]))
        if len(cache.tensors) == 5:
            K, V, Ks, Vs = cache.tensors[:4]
            K[o, :, i], V[o, :, i], Ks[o, :, i], Vs[o, :, i] = 0x7F, 0xFF, 255, 255
        else:
            for x in cache.tensors[:2]:
                x[o, :, i] = float("nan")
        if table is not None:
            for pg in range(table.shape[1]):
                if not seen[pg * page:(pg + 1) * page].any():
                    table[b, pg] = (-7, 1 << 30)[pg % 2]


def check(Q, O, LSE, keys, scale, bits, only=None):
    """keys(b, h, t) -> K, V fp64 that query t of request b sees on kv-head h.  Tolerances: O is bf16 (half a step: 2^-8
    of the value); a weight is off by at most half a step of bf16, 2^-8 of itself, where it is held in 16 bits, or by
    2^-30 of the largest weight where three short terms underflow; scores and exponentials in fp32 add below 2^-13 (d
    products, |score| < 2^7).  A = sum p |v| carries the relative errors.  LSE: d products of |q k| in fp32, each
    partial sum off by 2^-23 of it, and the sum of the weights; with 8 bits, query values below 2^-13 of their row's
    maximum may be off by 2^-17 of that maximum."""
    B, H_q, T, d = Q.shape
    q, Og, Lg = (x.double().cpu().numpy() for x in (Q, O, LSE))
    H_kv = keys(0, None, None)
    G = H_q // H_kv
    worst = 0.0
    for b in range(B):
        for h in range(H_kv):
            for t in range(T):
                if only is not None and not only(b, h, t):
                    continue
                K, V = keys(b, h, t)
                qr, og, lg = q[b, h * G:(h + 1) * G, t], Og[b, h * G:(h + 1) * G, t], Lg[b, h * G:(h + 1) * G, t]
                o, lse, A = kv8.attention(qr, K, V, scale)
                if K.shape[0] == 0:
                    assert (og == 0).all() and (lg == -np.inf).all(), (b, h, t)
                    continue
                assert np.isfinite(og).all(), (b, h, t)
                tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -13) * A + K.shape[0] * 2.0 ** -30 * np.abs(V).max() + 1e-30
                bad = np.abs(og - o) / tol
                assert bad.max() <= 1.0, (b, h, t, float(bad.max()))
                worst = max(worst, float(bad.max()))
                s_abs = scale * (np.abs(qr) @ np.abs(K).T).max(1)
                ltol = 2.0 ** -18 * s_abs + 2.0 ** -20 * np.abs(lse) + 2.0 ** -16
                if bits == 8:
                    top = np.abs(qr).max(1, keepdims=True)
                    ltol = ltol + (scale * 2.0 ** -17 * ((np.abs(qr) < 2.0 ** -13 * top) * top) @ np.abs(K).T).max(1)
                assert (np.abs(lg - lse) <= ltol).all(), (b, h, t, float(np.abs(lg - lse).max()))
    return worst


def keys_of(cache, H_kv, lens, T, window, sinks, depth=None, decode=True, local=None):
    """keys() of check(); local(b, h, t) -> candidates' K, V that query t sees besides."""
    memo = {}

    def keys(b, h, t):
        if h is None:
            return H_kv
        if b not in memo:
            memo.clear()
            memo[b] = [history(cache, b, seen_by(p, lens[b], window, sinks))
                       for p in positions(lens[b], T, None if depth is None else depth[b], decode)]
        K, V = (x[h] for x in memo[b][t])
        if local is not None:
            k, v = local(b, h, t)
            K, V = np.concatenate([K, k]), np.concatenate([V, v])
        return K, V
    return keys


def step(ssb, bits, cache, Q, lens, window, sinks, scale=None, ctx=None, flags=0, kernel=None, stream=None):
    B, H_q, T, d = Q.shape
    own = ctx is None
    room = cache.desc.page_size * cache.desc.pages_per_req
    ctx = ctx or ssb.Context(B, H_q, cache.H_kv, d, T, 1, room, flags=flags)
    O = torch.full((B, H_q, T, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    LSE = torch.full((B, H_q, T), float("nan"), device=DEV)
    f = ctx.ss_decode8_window if bits == 8 else ctx.ss_decode_window
    f(Q, scale or d ** -0.5, cache, window, sinks, _i32(lens), O, LSE, stream)
    torch.cuda.synchronize()
    assert ctx.ss_poll_status() == (0, 0)
    if kernel:
        assert kernel in ctx.last_chunk_kernel(), ctx.last_chunk_kernel()
    if own:
        ctx.close()
    return O, LSE


def queries(gen, B, H_q, T, d, how="bhtd"):
    if how == "bthd":
        return torch.randn(B, T, H_q, d, generator=gen).bfloat16().to(DEV).transpose(1, 2)
    return torch.randn(B, H_q, T, d, generator=gen).bfloat16().to(DEV)


LENS = [0, 1, 5, 127, 128, 129, 300, 511, 512, 700]
SHAPES = [  # window, sinks
    (1, 0), (1, 4), (7, 3), (100, 0), (128, 4), (129, 128), (250, 1), (64, 300), (1000, 0), (2 ** 31 - 1, 2 ** 31 - 1),
]


@pytest.mark.parametrize("window,sinks", SHAPES)
@pytest.mark.parametrize("bits,page,d,G,order", [
    (16, 0, 64, 1, (0, 1, 2)), (16, 8, 128, 4, (0, 2, 1)), (16, 16, 64, 8, (0, 1, 2)), (16, 24, 128, 1, (0, 1, 2)),
    (16, 64, 128, 12, (0, 2, 1)), (16, 96, 64, 3, (1, 0, 2)), (16, 128, 128, 4, (0, 1, 2)), (16, 5, 64, 2, (0, 1, 2)), (16, 1, 128, 9, (0, 2, 1)),
    (8, 0, 128, 4, (0, 1, 2)), (8, 16, 64, 1, (0, 2, 1)), (8, 40, 128, 8, (0, 1, 2)), (8, 256, 64, 5, (0, 1, 2)), (8, 3, 128, 2, (0, 1, 2)),
])
def test_one_token(bits, page, d, G, order, window, sinks):
    """A decoding step over requests of all lengths; what is not seen is NaN, pages without a seen token are gone."""
    ssb = _ssb()
    H_kv, room = 2, 768
    B = len(LENS)
    g = _gen(window % 1000 + sinks % 1000 + page + d)
    cache = make(ssb, bits, B, H_kv, d, page, room, page + G, order)
    Q = queries(g, B, H_kv * G, 1, d, "bthd")
    hide(cache, LENS, 1, window, sinks, room)
    for flags in ((0, ssb.SS_FLAG_FORCE_SIMT) if bits == 16 and page in (16, 24) else (0,)):
        kernel = "simt" if flags or page in (1, 3, 5) else "tcgen05"
        O, LSE = step(ssb, bits, cache, Q, LENS, window, sinks, flags=flags, kernel=kernel)
        check(Q, O, LSE, keys_of(cache, H_kv, LENS, 1, window, sinks), d ** -0.5, bits)


@pytest.mark.parametrize("bits,page,d,G,T,window,sinks", [
    (16, 16, 128, 4, 2, 100, 4), (16, 0, 64, 2, 24, 33, 5), (16, 64, 128, 1, 17, 1000, 0), (16, 8, 64, 1, 200, 5, 0), (16, 32, 128, 5, 9, 1, 2),
    (16, 7, 64, 4, 6, 20, 3), (16, 128, 64, 3, 31, 128, 128), (16, 16, 128, 1, 300, 150, 7),
    (8, 16, 128, 4, 3, 90, 4), (8, 0, 64, 1, 130, 9, 1), (8, 48, 128, 8, 8, 256, 0), (8, 5, 64, 2, 7, 30, 2),
])
def test_pieces(bits, page, d, G, T, window, sinks):
    """Several of the newest tokens at a time, each behind its own window; lengths below T leave queries without a key."""
    ssb = _ssb()
    lens = [n for n in (0, 1, T - 1, T, T + 1, 129, 500, 640)]
    H_kv, B, room = 2, 8, 768
    g = _gen(T + window)
    cache = make(ssb, bits, B, H_kv, d, page, room, T)
    Q = queries(g, B, H_kv * G, T, d)
    hide(cache, lens, T, window, sinks, room)
    O, LSE = step(ssb, bits, cache, Q, lens, window, sinks)
    check(Q, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks), d ** -0.5, bits)


def _tree(gen, B, T):
    """Parents before children: depths, ancestor bits (themselves among them)."""
    depth, bits = np.zeros((B, T), dtype=np.int64), np.zeros((B, T, T), dtype=bool)
    for b in range(B):
        bits[b, 0, 0] = True
        for i in range(1, T):
            par = int(torch.randint(0, i, (1,), generator=gen))
            depth[b, i] = depth[b, par] + 1
            bits[b, i] = bits[b, par]
            bits[b, i, i] = True
    return depth.tolist(), bits


def _words(bits):
    B, T, _ = bits.shape
    out = np.zeros((B, T, (T + 63) // 64), dtype=np.uint64)
    for j in range(T):
        out[:, :, j // 64] |= bits[:, :, j].astype(np.uint64) << np.uint64(j % 64)
    return torch.from_numpy(out.view(np.int64)).to(DEV)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("bits,page,d,G,T,window,sinks", [
    (16, 16, 128, 4, 8, 100, 4), (16, 0, 64, 2, 5, 1000, 0), (16, 128, 128, 8, 8, 260, 128), (16, 24, 64, 1, 64, 40, 1), (16, 3, 128, 1, 4, 9, 2),
    (8, 32, 128, 4, 6, 300, 16), (8, 0, 64, 5, 8, 17, 0), (8, 9, 64, 1, 3, 60, 4),
])
def test_rounds(bits, page, d, G, T, window, sinks, tree):
    ssb = _ssb()
    lens = [0, 3, 128, 417, 700]
    B, H_kv, room = len(lens), 2, 720
    g = _gen(T + window + page)
    cache = make(ssb, bits, B, H_kv, d, page, room, 5)
    Q, K_loc, V_loc = queries(g, B, H_kv * G, T, d), queries(g, B, H_kv, T, d), queries(g, B, H_kv, T, d)
    depth, seen = _tree(g, B, T) if tree else (None, np.tril(np.ones((T, T), dtype=bool))[None].repeat(B, 0))
    hide(cache, lens, T, window, sinks, room, depth, False)
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, cache.desc.page_size * cache.desc.pages_per_req)
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    ctx.ss_verify_begin(Q, d ** -0.5)
    chunk = ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window
    chunk(cache, window, sinks, _i32(lens), _i32(depth))
    ctx.ss_verify_local(K_loc, V_loc, ssb.SS_MASK_TREE_BITS if tree else ssb.SS_MASK_CHAIN, _words(seen) if tree else None)
    ctx.ss_verify_finalize(O, LSE)
    assert ctx.ss_poll_status() == (0, 0)
    kl, vl = K_loc.double().cpu().numpy(), V_loc.double().cpu().numpy()
    local = lambda b, h, t: (kl[b, h][seen[b, t]], vl[b, h][seen[b, t]])
    check(Q, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks, depth, False, local), d ** -0.5, bits)
    ctx.close()


# The three ways units meet CTAs: a few units long enough to be cut, clusters of several sizes, whole units.
FORMS = [
    ("tcgen05", 1, 1, 8500, 4, (9000,)), ("tcgen05", 3, 1, 8800, 130, (0, 9000, 4100)), ("tcgen05", 1, 2, 2 ** 31 - 1, 0, (8999,)),
    ("tcgen05-cluster", 1, 1, 1000, 4, (9000,)), ("tcgen05-cluster", 1, 1, 250, 0, (9000,)), ("tcgen05-cluster", 4, 2, 300, 3, (0, 9, 400, 9000)),
    ("tcgen05-cluster", 100, 2, 200, 4, None), ("tcgen05-whole", 250, 2, 300, 20, None), ("tcgen05-whole", 300, 3, 100, 0, None),
]


@pytest.mark.parametrize("form,B,H_kv,window,sinks,lens", FORMS)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d,G,T", [(128, 4, 1), (64, 2, 1), (64, 5, 5), (128, 8, 4)])
def test_forms(form, B, H_kv, window, sinks, lens, bits, d, G, T):
    ssb = _ssb()
    g = _gen(B + window % 1000 + d)
    room = 9024 if lens else 704
    lens = list(lens) if lens else [int(x) for x in torch.randint(0, 700, (B,), generator=g)]
    cache = make(ssb, bits, B, H_kv, d, 32, room, B)
    Q = queries(g, B, H_kv * G, T, d)
    if B < 10:
        hide(cache, lens, T, window, sinks, room)
    O, LSE = step(ssb, bits, cache, Q, lens, window, sinks, kernel="tcgen05")
    ctx = ssb.Context(B, H_kv * G, H_kv, d, T, 1, room)
    O2, LSE2 = step(ssb, bits, cache, Q, lens, window, sinks, ctx=ctx)
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2)       # the same bits again
    if T == 1:                                                 # (with more rows the estimate may take another form)
        assert ctx.last_chunk_kernel().endswith(form), ctx.last_chunk_kernel()
    ctx.close()
    only = None if B < 10 else (lambda b, h, t: b % 37 == 0 or lens[b] < 3)
    check(Q, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks), d ** -0.5, bits, only)


@pytest.mark.parametrize("form,B,H_kv,window,sinks,lens", FORMS)
@pytest.mark.parametrize("bits,d,G,T", [(16, 128, 4, 8), (16, 64, 2, 3), (8, 128, 4, 6), (8, 64, 8, 2)])
def test_forms_in_rounds(form, B, H_kv, window, sinks, lens, bits, d, G, T):
    """The forms as chunks: alone, and behind another chunk of the same round with the sets folded."""
    ssb = _ssb()
    g = _gen(B + window % 1000 + d + 1)
    room = 9024 if lens else 704
    lens = list(lens) if lens else [int(x) for x in torch.randint(0, 700, (B,), generator=g)]
    cache = make(ssb, bits, B, H_kv, d, 16, room, B)
    Q, K_loc, V_loc = queries(g, B, H_kv * G, T, d), queries(g, B, H_kv, T, d), queries(g, B, H_kv, T, d)
    if B < 10:
        hide(cache, lens, T, window, sinks, room, None, False)
    more = queries(g, B, H_kv, 40, d), queries(g, B, H_kv, 40, d)
    n = _i32(lens)
    kl, vl, km, vm = (x.double().cpu().numpy() for x in (K_loc, V_loc) + more)
    only = None if B < 10 else (lambda b, h, t: b % 53 == 0 or lens[b] < 3)
    for flags in (0, ssb.SS_FLAG_OVERLAP_CHUNKS):
        ctx = ssb.Context(B, H_kv * G, H_kv, d, T, T, room, max_chunks=2, flags=flags)
        chunk = ctx.ss_verify_chunk8_window if bits == 8 else ctx.ss_verify_chunk_window
        for behind in (0, 1, 2):                               # other chunks in front: 2 fill the sets, which are folded
            O, LSE = torch.full_like(Q, float("nan")), torch.full(Q.shape[:3], float("nan"), device=DEV)
            ctx.ss_verify_begin(Q, d ** -0.5)
            for _ in range(behind):
                ctx.ss_verify_chunk(*more)
            chunk(cache, window, sinks, n)
            ctx.ss_verify_local(K_loc, V_loc)
            ctx.ss_verify_finalize(O, LSE)
            assert ctx.ss_poll_status() == (0, 0)

            def local(b, h, t):
                k, v = [km[b, h]] * behind + [kl[b, h, : t + 1]], [vm[b, h]] * behind + [vl[b, h, : t + 1]]
                return np.concatenate(k), np.concatenate(v)
            check(Q, O, LSE, keys_of(cache, H_kv, lens, T, window, sinks, None, False, local), d ** -0.5, bits, only)
        ctx.close()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("kernel", ["tcgen05", "simt"])
def test_states_and_mixed_chunks(bits, kernel):
    """Window chunks beside each other, beside plain and whole-history chunks, exported in between and imported elsewhere."""
    ssb = _ssb()
    B, H_kv, G, d, T, room, page = 3, 2, 4, 128, 4, 2048, 16 if kernel == "tcgen05" else 5
    lens, lens8 = [900, 0, 2040], [100, 300, 0]
    g = _gen(3)
    c16, c8 = make(ssb, 16, B, H_kv, d, page, room, 1), make(ssb, 8, B, H_kv, d, page, room, 2)
    Q, K_loc, V_loc = queries(g, B, H_kv * G, T, d), queries(g, B, H_kv, T, d), queries(g, B, H_kv, T, d)
    K, V = queries(g, B, H_kv, 64, d), queries(g, B, H_kv, 64, d)
    one, two = (ssb.Context(B, H_kv * G, H_kv, d, T, T, room + page, max_chunks=3) for _ in range(2))
    rows = B * H_kv * G * T
    ml, a = torch.empty(rows, 2, device=DEV), torch.empty(rows, d, device=DEV)
    O, LSE = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
    one.ss_verify_begin(Q, d ** -0.5)
    one.ss_verify_chunk_window(c16, 500, 4, _i32(lens))
    one.ss_verify_chunk8(c8, _i32(lens8))
    one.ss_verify_chunk8_window(c8, 70, 2, _i32(lens))
    one.ss_verify_export_state(ml, a)
    one.ss_verify_abort()
    two.ss_verify_begin(Q, d ** -0.5)
    two.ss_verify_chunk(K, V)
    two.ss_verify_chunk_window(c16, 33, 0, _i32(lens8))
    two.ss_verify_import_state(ml, a)
    two.ss_verify_local(K_loc, V_loc)
    two.ss_verify_finalize(O, LSE)
    assert one.ss_poll_status() == (0, 0) and two.ss_poll_status() == (0, 0)
    parts = [keys_of(c16, H_kv, lens, T, 500, 4, None, False), keys_of(c8, H_kv, lens8, T, 10 ** 6, 0, None, False),
             keys_of(c8, H_kv, lens, T, 70, 2, None, False), keys_of(c16, H_kv, lens8, T, 33, 0, None, False)]
    kl, vl, km, vm = (x.double().cpu().numpy() for x in (K_loc, V_loc, K, V))

    def keys(b, h, t):
        if h is None:
            return H_kv
        kv = [f(b, h, t) for f in parts] + [(km[b, h], vm[b, h]), (kl[b, h, : t + 1], vl[b, h, : t + 1])]
        return np.concatenate([x[0] for x in kv]), np.concatenate([x[1] for x in kv])
    check(Q, O, LSE, keys, d ** -0.5, 8)
    one.close()
    two.close()
