"""Rotary positions, appending to a cache and attention over a window, at sizes they are used at.

Rotation.  Pair i of a row (its elements i and i + rot / 2, or 2 i and 2 i + 1 in the interleaved layout; elements from
`rot` on stay) at position p on the pair's axis turns by p * f_i.  A token has one position, or one for each axis.

Append.  Rows of K, rotated, and of V become tokens of a cache; the rows of Q that go with them are rotated as well.  A
cache is paged ([pages, H_kv, page, d] with a table of page ids per request) or dense ([B, H_kv, tokens, d]), in bf16 or
in 8 bits: d codes in e4m3 and an exponent e per row, the smallest integer in [-32, 80] with max|x| <= 448 * 2^e, held as
the byte e + 127; a value is code * 2^e.  The rows that are held in 8 bits are the rotated ones in bf16.

Window.  A query at position p sees token j of its request when j <= p and (j < sinks or p - j < window).  The queries
are the newest tokens of the cache ("decode"), or candidates behind it that see one another along a chain or a tree
("verify").
"""
import math

import numpy as np
import torch

own = False

# Most values of a drawn case: rows of an append or a rotation, visible keys of an attention (each times d and heads).
_MOST_ROWS = 1 << 27
_MOST_KEYS = 1 << 27


def _rows_case(name, kind, B, H_q, H_kv, d, lo, hi, page=0, bits=16, rot=None, axes=1, inter=False, pick=False, q=True):
    c = dict(kind=kind, B=B, H_q=H_q, H_kv=H_kv, d=d, lo=lo, hi=hi, page=page, bits=bits, rot=d if rot is None else rot,
             axes=axes, inter=inter, pick=pick, q=q)
    return c if name is None else c | {"name": name}


def _attend_case(name, kind, B, H_q, H_kv, d, T_q, lo, hi, window, sinks, page=0, bits=16, tree=False, freed=False):
    c = dict(kind=kind, B=B, H_q=H_q, H_kv=H_kv, d=d, T_q=T_q, lo=lo, hi=hi, window=window, sinks=sinks, page=page,
             bits=bits, tree=tree, freed=freed)
    return c if name is None else c | {"name": name}


def listed():
    """For `rotate` and `append`, lo..hi is how many rows a request's call carries (`pick`: accepted ones out of hi
    candidates; rot = 0: rotated already); for the others, how many tokens a request has in the cache (`freed`: the pages
    between the sinks and the window have been given back)."""
    return [
        # the candidates of a Qwen3-8B-shaped round, before its attention
        _rows_case("rotate_candidates", "rotate", 16, 32, 8, 128, 8, 8),
        # a video prompt: time, height and width
        _rows_case("rotate_video", "rotate", 2, 32, 8, 128, 8192, 8192, axes=3),
        # decoding: every request's newest token joins the pages, its query is rotated on the way
        _rows_case("append_new_tokens", "append", 64, 32, 8, 128, 1, 1, page=16),
        # the end of a round: the accepted ones of 8 candidates, rotated before the attention, join the pages
        _rows_case("append_accepted", "append", 32, 32, 8, 128, 1, 8, page=64, rot=0, pick=True, q=False),
        # prompts of a ragged batch, written before their attention
        _rows_case("append_prompts", "append", 8, 32, 8, 128, 4001, 8192, page=64),
        # the same into a cache of 8 bits, a smaller head, rotated in part, pairs side by side, three axes
        _rows_case("append_prompts_8bit", "append", 4, 16, 4, 64, 700, 6007, page=32, bits=8, rot=32, axes=3, inter=True),
        # one short request on a small model: nothing but latency
        _attend_case("decode_tiny", "decode", 1, 4, 1, 64, 1, 1024, 1024, 256, 4, page=16),
        # a batch of long histories through a layer with a window
        _attend_case("decode_batch", "decode", 16, 32, 8, 128, 1, 32768, 32768, 4096, 4, page=64, freed=True),
        # many requests of all lengths, short window, small pages
        _attend_case("decode_ragged", "decode", 64, 32, 8, 128, 1, 37, 16384, 1024, 16, page=16, freed=True),
        # a prompt's last piece: 24 tokens at a time against a dense cache
        _attend_case("decode_piece", "decode", 3, 8, 2, 64, 24, 900, 5003, 1000, 5),
        # the Qwen3-8B-shaped round of 8 candidates through a layer with a window
        _attend_case("verify_batch", "verify", 16, 32, 8, 128, 8, 32768, 32768, 8192, 4, page=128, freed=True),
        # a tree of candidates over a ragged cache of 8 bits
        _attend_case("verify_tree_8bit", "verify", 24, 32, 8, 128, 6, 3000, 32768, 4096, 128, page=32, bits=8, tree=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "decode", "decode", "verify"])
    d = rng.choice([64, 128])
    H_kv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    page = rng.choice([0, 8, 16, 32, 64, 128])
    bits = rng.choice([16, 16, 8])
    if kind in ("rotate", "append"):
        axes = rng.choice([1, 1, 3])
        rot = rng.choice([d, d, d // 2, d // 4])
        inter, q = rng.random() < 0.3, kind == "rotate" or rng.random() < 0.6
        pick = kind == "append" and rng.random() < 0.3
        if pick:
            q, rot, axes = False, rng.choice([0, d]), 1
        hi = rng.randint(2, 8) if pick else _log_int(rng, 1, 16384)
        B = _log_int(rng, 1, max(1, min(64, _MOST_ROWS // (hi * (H_kv * G + H_kv) * d))))
        lo = hi if kind == "rotate" else max(1, int(hi * rng.choice([1.0, 0.5, 0.1])))
        if kind == "rotate":
            page, bits = 0, 16
        return _rows_case(None, kind, B, H_kv * G, H_kv, d, lo, hi, page, bits, rot, axes, inter, pick, q)
    T_q = rng.randint(2, 8) if kind == "verify" else rng.choice([1, 1, 1, rng.randint(2, 24)])
    window, sinks = _log_int(rng, 32, 8192), rng.choice([0, 1, 4, 16, 128])
    hi = max(T_q, _log_int(rng, 16, 32768))
    most = _MOST_KEYS // (min(hi, window + sinks + T_q) * H_kv * d * max(1, G * T_q // 32))
    B = _log_int(rng, 1, max(1, min(64, most)))
    lo = max(T_q, int(hi * rng.choice([1.0, 0.5, 0.1])))
    return _attend_case(None, kind, B, H_kv * G, H_kv, d, T_q, lo, hi, window, sinks, page, bits,
                        kind == "verify" and rng.random() < 0.5, page > 0 and rng.random() < 0.5)


def _lengths(c):
    """Lengths of the requests: spread over lo..hi, in no order."""
    span = c["hi"] - c["lo"]
    return [c["lo"] + int(round(span * ((0.37 + b * 0.6180339887498949) % 1.0))) for b in range(c["B"])]


def _frequencies(c):
    """The angle of each pair per position, and its axis (the pairs of an axis side by side)."""
    n = c["rot"] // 2
    f = [1e6 ** (-i / n) for i in range(n)]
    return f, [min(i * c["axes"] // n, c["axes"] - 1) for i in range(n)]


def _room(c):
    """Tokens that the cache holds for a request."""
    top = c["hi"] + (64 if c["kind"] == "append" else 0)
    return -(-top // c["page"]) * c["page"] if c["page"] else -(-top // 8) * 8


def _normal(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _power(e):
    """2^e as fp32, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x):
    """fp32 rows -> (codes as float8, exponent bytes)."""
    mag = x.abs().amax(-1)
    m, ex = torch.frexp(mag)                                   # mag = m * 2^ex, m in [0.5, 1)
    e = torch.where(m > 0.875, ex - 8, ex - 9)                 # 448 = 0.875 * 2^9
    e = torch.where(mag == 0, torch.full_like(e, -32), e).clamp(-32, 80)
    y = x * _power(-e).unsqueeze(-1)
    return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _decode(codes, scale):
    return codes.view(torch.float8_e4m3fn).float() * _power(scale.to(torch.int32) - 127).unsqueeze(-1)


def _caches(c, gen, live):
    """Cache buffers of random rows.  `live` [B, pages]: which pages are there; the table's other entries are -1."""
    B, H_kv, d, page = c["B"], c["H_kv"], c["d"], c["page"]
    room = _room(c)
    outer, tokens, table = B, room, None
    if page:
        n = int(live.sum())
        outer, tokens = n + 3, page
        ids = torch.randperm(outer, generator=gen, device="cuda")[:n].to(torch.int32)
        table = torch.full((B, room // page), -1, dtype=torch.int32, device="cuda")
        table[live] = ids
    out = {"table": table, "K_scale": None, "V_scale": None}
    for name in ("K", "V"):
        x = torch.empty(outer, H_kv, tokens, d, dtype=torch.uint8 if c["bits"] == 8 else torch.bfloat16, device="cuda")
        scale = torch.empty(outer, H_kv, tokens, dtype=torch.uint8, device="cuda") if c["bits"] == 8 else None
        step = max(1, (1 << 26) // (H_kv * tokens * d))
        for i in range(0, outer, step):
            y = _normal(gen, (min(step, outer - i), H_kv, tokens, d))
            if name == "K":
                y[..., :: d // 4] *= 4.0                       # a few channels of K stand out
            else:
                y *= torch.exp(_normal(gen, y.shape[:3]) * 0.5).unsqueeze(-1)
            if c["bits"] == 8:
                q, scale[i:i + step] = _encode(y.bfloat16().float())
                x[i:i + step] = q.view(torch.uint8)
            else:
                x[i:i + step] = y
        out[name], out[name + "_scale"] = x, scale
    return out


def _spoil(c, s, n):
    """Behind a request's last token (n [B, 1]): anything, NaN too."""
    tok = torch.arange(_room(c), device="cuda")
    b, t = (tok >= n).nonzero(as_tuple=True)
    if c["page"]:
        o, i = s["table"][b, t // c["page"]].long(), t % c["page"]
        o, i = o[o >= 0], i[o >= 0]
    else:
        o, i = b, t
    for name in ("K", "V"):
        s[name][o, :, i] = 0x7F if c["bits"] == 8 else math.nan


def _prepare_rows(c, gen, s):
    B, H_q, H_kv, d, T = c["B"], c["H_q"], c["H_kv"], c["d"], c["hi"]
    lens = _lengths(c)
    s["K_new"] = _normal(gen, (B, H_kv, T, d)).bfloat16()
    s["Q"] = _normal(gen, (B, H_q, T, d)).bfloat16() if c["q"] else None
    s["Q_out"] = torch.zeros_like(s["Q"]) if c["q"] else None
    if c["rot"]:
        f, axis = _frequencies(c)
        s["freq"] = torch.tensor(f, dtype=torch.float64, device="cuda")
        s["axis"] = torch.tensor(axis, device="cuda")
    s["pos"] = None
    if c["axes"] > 1:                                          # frames of 24 x 32 patches
        t = torch.arange(T, device="cuda")
        pos = torch.stack([t // 768, t // 32 % 24, t % 32][: c["axes"]]).unsqueeze(1).expand(-1, B, -1)
        start = torch.randint(0, 4096, (1, B, 1), generator=gen, device="cuda")
        s["pos"] = (pos + start).to(torch.int32).contiguous()
    if c["kind"] == "rotate":
        s["off"] = torch.randint(0, 1 << 17, (B,), generator=gen, device="cuda").to(torch.int32)
        s["K_out"] = torch.zeros_like(s["K_new"])
        return
    room = _room(c)
    live = torch.ones(B, room // c["page"], dtype=torch.bool, device="cuda") if c["page"] else None
    s |= _caches(c, gen, live)
    s["V_new"] = (_normal(gen, (B, H_kv, T, d)) * 0.5).bfloat16()
    s["cnt"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["off"] = torch.tensor([(13 * b + 5) % (room - T + 1) for b in range(B)], dtype=torch.int32, device="cuda")
    s["idx"] = None
    if c["pick"]:                                              # a path through the candidates, in order
        pick = torch.rand(B, T, generator=gen, device="cuda").argsort(1)
        keep = torch.arange(T, device="cuda") < s["cnt"].unsqueeze(1)
        pick = torch.where(keep, pick, torch.full_like(pick, T)).sort(1).values
        s["idx"] = pick.clamp(max=T - 1).to(torch.int32).contiguous()


def _prepare_attend(c, gen, s):
    B, H_q, H_kv, d, T = c["B"], c["H_q"], c["H_kv"], c["d"], c["T_q"]
    lens = _lengths(c)
    n = torch.tensor(lens, device="cuda").unsqueeze(1)
    live = None
    if c["page"]:
        first = torch.arange(_room(c) // c["page"], device="cuda") * c["page"]
        live = (first < n).clone()
        if c["freed"]:
            from_ = n + (1 if c["kind"] == "verify" else 1 - T) - c["window"]
            live &= (first < c["sinks"]) | (first + c["page"] > from_)
    s |= _caches(c, gen, live)
    _spoil(c, s, n)
    u = torch.sign(_normal(gen, (H_kv, d)))                    # the direction that every query shares
    q = _normal(gen, (B, H_kv, H_q // H_kv, T, d)) + 0.5 * u.view(1, H_kv, 1, 1, d)
    s["Q"] = q.reshape(B, H_q, T, d).bfloat16()
    if c["sinks"]:                                             # the first token draws attention, its V is small
        first = s["table"][:, 0].long() if c["page"] else torch.arange(B, device="cuda")
        if c["bits"] == 8:
            code, e = _encode(2.0 * u)
            s["K"][first, :, 0], s["K_scale"][first, :, 0] = code.view(torch.uint8), e
            s["V_scale"][first, :, 0] -= 3
        else:
            s["K"][first, :, 0] = (2.0 * u).bfloat16()
            s["V"][first, :, 0] /= 8.0
    s["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["O"] = torch.empty_like(s["Q"])
    s["LSE"] = torch.empty(B, H_q, T, device="cuda")
    s["depth"] = s["bits"] = None
    if c["kind"] == "verify":
        s["K_loc"] = _normal(gen, (B, H_kv, T, d)).bfloat16()
        s["V_loc"] = _normal(gen, (B, H_kv, T, d)).bfloat16()
        if c["tree"]:                                          # node i hangs on one of the nodes before it
            par = (torch.rand(B, T, generator=gen, device="cuda") * torch.arange(T, device="cuda")).long().tolist()
            depth, bits = [], []
            for b in range(B):
                deep, seen = [0], [1]
                for i in range(1, T):
                    deep.append(deep[par[b][i]] + 1)
                    seen.append(seen[par[b][i]] | 1 << i)
                depth.append(deep)
                bits.append(seen)
            s["depth"] = torch.tensor(depth, dtype=torch.int32, device="cuda")
            s["bits"] = torch.tensor(bits, dtype=torch.int64, device="cuda").unsqueeze(2).contiguous()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    s = {"case": c, "scale": c["d"] ** -0.5}
    rows = c["kind"] in ("rotate", "append")
    (_prepare_rows if rows else _prepare_attend)(c, gen, s)
    if own:
        from paper_2609_33184_b200 import binding as ss
        T = 1 if rows else c["T_q"]
        s["ctx"] = ss.Context(c["B"], c["H_q"], c["H_kv"], c["d"], T, T, _room(c))
        if c["kind"] != "rotate":
            s["cache"] = (ss.Cache8(s["K"], s["V"], s["K_scale"], s["V_scale"], s["table"]) if c["bits"] == 8
                          else ss.Cache16(s["K"], s["V"], s["table"]))
        if rows:
            s["rope"] = ss.Rope(*_frequencies(c), n_axes=c["axes"], interleaved=c["inter"]) if c["rot"] else None
    return s


def _turn(s, x, pos):
    """Rows x [B, H, T, d] at positions [axes, B, T] -> rotated, fp32."""
    c = s["case"]
    x, rot = x.float(), c["rot"]
    angle = pos[s["axis"]].permute(1, 2, 0).double() * s["freq"]                     # [B, T, pairs]
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["inter"] else (x[..., : rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, v], -1).flatten(-2) if c["inter"] else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rows(s):
    c = s["case"]
    B, T = c["B"], c["hi"]
    k = torch.arange(T, device="cuda")
    src = k.expand(B, T) if s.get("idx") is None else s["idx"].long()
    K = s["K_new"]
    if s.get("idx") is not None:
        K = torch.gather(K, 2, src[:, None, :, None].expand(-1, c["H_kv"], -1, c["d"]))
    Q = s["Q"]
    if c["rot"]:
        pos = (s["off"].long().unsqueeze(1) + k).unsqueeze(0) if s["pos"] is None else s["pos"]
        K = _turn(s, K, pos).bfloat16()
        Q = None if Q is None else _turn(s, Q, pos).bfloat16()
    if c["kind"] == "rotate":
        return Q, K
    live = k.unsqueeze(0) < s["cnt"].unsqueeze(1)
    b, k = live.nonzero(as_tuple=True)
    tok = s["off"].long()[b] + k
    o, i = (s["table"].long()[b, tok // c["page"]], tok % c["page"]) if c["page"] else (b, tok)
    for name, x in (("K", K[b, :, k]), ("V", s["V_new"][b, :, src[b, k]])):
        if c["bits"] == 8:
            q, e = _encode(x.float())
            s[name][o, :, i], s[name + "_scale"][o, :, i] = q.view(torch.uint8), e
        else:
            s[name][o, :, i] = x
    if Q is not None:
        s["Q_out"] = torch.where(live[:, None, :, None], Q, s["Q_out"])
    return _cache_out(s)


def _cache_out(s):
    """The whole cache as the values that it stands for (8 bits: codes and powers of two), and the rotated queries."""
    out = [s["K"], s["V"]]
    if s["case"]["bits"] == 8:
        out = [x.view(torch.float8_e4m3fn) for x in out]
        out += [s[n].view(torch.float8_e8m0fnu) for n in ("K_scale", "V_scale")]
    return out if s["Q_out"] is None else out + [s["Q_out"]]


def _plain_attention(s):
    c = s["case"]
    B, H_q, H_kv, d, T, W = c["B"], c["H_q"], c["H_kv"], c["d"], c["T_q"], c["window"]
    n = s["len"].long().unsqueeze(1)                           # [B, 1]
    first = n if c["kind"] == "verify" else n - T              # position of query 0
    t = torch.arange(T, device="cuda").unsqueeze(0)
    pos = first + (t if s["depth"] is None else s["depth"].long())                   # [B, T]
    sinks = min(c["sinks"], c["hi"])
    span = min(W + T, c["hi"])                                 # tokens that some query has in its window
    near = (first + 1 - W).clamp(min=0) + torch.arange(span, device="cuda")
    tok = torch.cat([torch.arange(sinks, device="cuda").expand(B, sinks), near], 1)  # [B, U]
    there = tok < n
    there[:, sinks:] &= near >= sinks
    seen = there.unsqueeze(1) & (tok.unsqueeze(1) <= pos.unsqueeze(2))
    seen &= (tok.unsqueeze(1) < sinks) | (pos.unsqueeze(2) - tok.unsqueeze(1) < W)   # [B, T, U]
    tok = torch.where(there, tok, torch.zeros_like(tok))
    o, i = tok, tok
    if c["page"]:
        o, i = torch.gather(s["table"].long(), 1, tok // c["page"]).clamp(min=0), tok % c["page"]
    else:
        o = torch.arange(B, device="cuda").unsqueeze(1).expand_as(tok)

    def rows(name):
        x = s[name][o, :, i]                                   # [B, U, H_kv, d]
        x = _decode(x, s[name + "_scale"][o, :, i]) if c["bits"] == 8 else x.float()
        return torch.where(there[:, :, None, None], x, torch.zeros((), device="cuda")).transpose(1, 2)

    G = H_q // H_kv
    none = torch.full((), -math.inf, device="cuda")
    q = s["Q"].float().reshape(B, H_kv, G * T, d) * s["scale"]
    score = torch.where(seen.repeat(1, G, 1).unsqueeze(1), q @ rows("K").transpose(2, 3), none)
    V = rows("V")
    if c["kind"] == "verify":
        if s["bits"] is None:
            mask = (t <= t.transpose(0, 1)).expand(B, T, T)
        else:
            mask = (s["bits"] >> t.unsqueeze(0) & 1).bool()
        loc = torch.where(mask.repeat(1, G, 1).unsqueeze(1), q @ s["K_loc"].float().transpose(2, 3), none)
        score, V = torch.cat([score, loc], -1), torch.cat([V, s["V_loc"].float()], 2)
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = w.sum(-1, keepdim=True)
    out = torch.where(total > 0, w @ V / total, torch.zeros((), device="cuda"))
    lse = (top + torch.log(total)).reshape(B, H_q, T)
    return out.reshape(B, H_q, T, d).bfloat16(), lse


def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if own:
        ctx = s["ctx"]
        if kind == "rotate":
            ctx.ss_rope_rotate(s["rope"], s["Q"], s["K_new"], s["Q_out"], s["K_out"], pos=s["pos"], pos_off=s["off"])
            return s["Q_out"], s["K_out"]
        if kind == "append":
            append = ctx.ss_kv8_append if c["bits"] == 8 else ctx.ss_kv_append
            append(s["cache"], s["K_new"], s["V_new"], s["rope"], s["pos"], s["Q"], s["Q_out"], s["off"], s["cnt"], s["idx"])
            return _cache_out(s)
        if kind == "decode":
            decode = ctx.ss_decode8_window if c["bits"] == 8 else ctx.ss_decode_window
            decode(s["Q"], s["scale"], s["cache"], c["window"], c["sinks"], s["len"], s["O"], s["LSE"])
            return s["O"], s["LSE"]
        from paper_2609_33184_b200 import binding as ss
        ctx.ss_verify_begin(s["Q"], s["scale"])
        chunk = ctx.ss_verify_chunk8_window if c["bits"] == 8 else ctx.ss_verify_chunk_window
        chunk(s["cache"], c["window"], c["sinks"], s["len"], s["depth"])
        ctx.ss_verify_local(s["K_loc"], s["V_loc"], ss.SS_MASK_TREE_BITS if c["tree"] else ss.SS_MASK_CHAIN, s["bits"])
        ctx.ss_verify_finalize(s["O"], s["LSE"])
        return s["O"], s["LSE"]
    return _plain_rows(s) if kind in ("rotate", "append") else _plain_attention(s)


def work(case):
    c = case
    n, d, H_q, H_kv = sum(_lengths(c)), c["d"], c["H_q"], c["H_kv"]
    if c["kind"] in ("rotate", "append"):
        row = 2 * d if c["bits"] == 16 else d + 1
        turned = H_kv + (H_q if c["q"] else 0)
        byte = n * turned * 4 * d if c["kind"] == "rotate" else n * (2 * H_kv * (2 * d + row) + (H_q * 4 * d if c["q"] else 0))
        return {"bytes": byte, "flops": n * turned * 3 * c["rot"] + n * 2 * H_kv * d}
    T, W, S = c["T_q"], c["window"], c["sinks"]
    R = H_q // H_kv * T
    keys = pairs = 0
    for m in _lengths(c):
        first = m if c["kind"] == "verify" else m - T
        lo = max(0, first + 1 - W)
        keys += m - lo + min(S, lo)
        pairs += (m - lo + min(S, lo)) * R
    row = 2 * d if c["bits"] == 16 else d + 1
    rows = c["B"] * H_q * T
    byte, flop = keys * H_kv * 2 * row + rows * (4 * d + 4), 4 * pairs * H_kv * d
    if c["kind"] == "verify":
        byte += c["B"] * H_kv * T * 4 * d
        flop += 2 * rows * (T + 1) * d
    return {"bytes": byte, "flops": flop}


def _to_bf16(x):
    """Nearest bf16 values (even of two equally near ones) of an fp64 array of ordinary magnitudes."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def _exact_code(x):
    """A row's values in 64 bits -> (the e4m3 values of its codes, its scale), from the format's definition."""
    top = np.abs(x).max(-1)
    e = np.full(top.shape, -32, dtype=np.int64)
    some = top > 0
    e[some] = np.clip(np.ceil(np.log2(top[some] / 448.0) - 1e-13), -32, 80).astype(np.int64)
    e += (top > 448.0 * np.exp2(e.astype(np.float64))) & (e < 80)
    y = np.clip(x * np.exp2(-e.astype(np.float64))[..., None], -448.0, 448.0)
    grain = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 1e-300))), -6.0) - 3.0)
    return np.rint(y / grain) * grain, np.exp2(e.astype(np.float64))


def _exact_rows(c, s):
    B, H_kv, d, T, rot = c["B"], c["H_kv"], c["d"], c["hi"], c["rot"]
    lens = [T] * B if c["kind"] == "rotate" else _lengths(c)
    if sum(lens) * (H_kv + c["H_q"] * c["q"]) * d > (1 << 28):
        return None
    host = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
    K, Q, off = host(s["K_new"]), host(s["Q"]), s["off"].tolist()
    pos = None if s["pos"] is None else s["pos"].cpu().numpy()
    f, axis = _frequencies(c) if rot else ([], [])
    half = rot // 2
    one, two = (np.arange(half) * 2, np.arange(half) * 2 + 1) if c["inter"] else (np.arange(half), np.arange(half) + half)

    def turned(x, b, n):
        x = x.copy()
        if rot:
            at = np.stack([off[b] + np.arange(n)] * half if pos is None else [pos[a, b, :n] for a in axis], 1).astype(np.float64)
            z = (x[..., one] + 1j * x[..., two]) * np.exp(1j * (at * np.array(f)))
            x[..., one], x[..., two] = z.real, z.imag
        return x

    if c["kind"] == "rotate":
        return np.stack([turned(Q[b], b, T) for b in range(B)]), np.stack([turned(K[b], b, T) for b in range(B)])
    V = host(s["V_new"])
    out = {n: host(s[n].view(torch.float8_e4m3fn) if c["bits"] == 8 else s[n]) for n in ("K", "V")}
    scale = {n: host(s[n + "_scale"].view(torch.float8_e8m0fnu)) for n in ("K", "V")} if c["bits"] == 8 else None
    Q_out = host(s["Q_out"])
    for b, n in enumerate(lens):
        src = np.arange(n) if s["idx"] is None else s["idx"][b, :n].cpu().numpy()
        tok = off[b] + np.arange(n)
        o, i = (s["table"][b].cpu().numpy()[tok // c["page"]], tok % c["page"]) if c["page"] else (np.full(n, b), tok)
        for name, x in (("K", turned(K[b][:, src], b, n)), ("V", V[b][:, src])):
            x = x.transpose(1, 0, 2)
            if c["bits"] == 8:
                out[name][o, :, i], scale[name][o, :, i] = _exact_code(_to_bf16(x))
            else:
                out[name][o, :, i] = x
        if Q is not None:
            Q_out[b, :, :n] = turned(Q[b, :, :n], b, n)
    got = [out["K"], out["V"]] + ([scale["K"], scale["V"]] if scale else [])
    return got if Q_out is None else got + [Q_out]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("rotate", "append"):
        return _exact_rows(c, s)
    B, H_q, H_kv, d, T, page = c["B"], c["H_q"], c["H_kv"], c["d"], c["T_q"], c["page"]
    G = H_q // H_kv
    O = torch.zeros(B, H_kv, G, T, d, dtype=torch.float64)
    L = torch.zeros(B, H_kv, G, T, dtype=torch.float64)
    # in 64 bits on the device, one request at a time
    for b, n in enumerate(_lengths(c)):
        first = n if c["kind"] == "verify" else n - T
        pos = [first + (t if s["depth"] is None else int(s["depth"][b, t])) for t in range(T)]
        j = torch.tensor(sorted(set(range(min(n, c["sinks"]))) | set(range(max(0, first + 1 - c["window"]), n))), device="cuda")
        o, i = (s["table"][b, j // page].long(), j % page) if page else (torch.full_like(j, b), j)
        kv = []
        for name in ("K", "V"):
            x = s[name][o, :, i].transpose(0, 1)               # [H_kv, keys, d]
            if c["bits"] == 8:
                q, e = x.to(torch.int16), s[name + "_scale"][o, :, i].transpose(0, 1).double()
                field, frac = (q >> 3) & 15, (q & 7).double()
                val = torch.where(field == 0, frac * 2.0 ** -9, (1.0 + frac / 8.0) * torch.exp2(field.double() - 7.0))
                x = torch.where(q >= 128, -val, val) * torch.exp2(e - 127.0).unsqueeze(-1)
            kv.append(x.double())
        at = torch.tensor(pos, device="cuda").unsqueeze(1)
        hide = (j > at) | ((j >= c["sinks"]) & (at - j >= c["window"]))              # [T, keys]
        for h in range(H_kv):
            q = s["Q"][b, h * G:(h + 1) * G].double()          # [G, T, d]
            a = torch.einsum("gtd,nd->gtn", q, kv[0][h]).mul(s["scale"]).masked_fill(hide, -math.inf)
            v = kv[1][h]
            if c["kind"] == "verify":
                near = torch.einsum("gtd,nd->gtn", q, s["K_loc"][b, h].double()) * s["scale"]
                for t in range(T):
                    seen = (1 << (t + 1)) - 1 if s["bits"] is None else int(s["bits"][b, t, 0])
                    near[:, t, [k for k in range(T) if not seen >> k & 1]] = -math.inf
                a, v = torch.cat([a, near], -1), torch.cat([v, s["V_loc"][b, h].double()])
            L[b, h] = torch.logsumexp(a, -1).cpu()
            O[b, h] = torch.einsum("gtn,nd->gtd", torch.nan_to_num(torch.softmax(a, -1)), v).cpu()
    return O.reshape(B, H_q, T, d), L.reshape(B, H_q, T)
