"""The 8-bit KV cache's operators at sizes they are used at: writing bf16 rows into the cache, reading them back,
attention of the newest tokens over the cache, and a verification round over it.

Format of a cache row (one token of one kv-head, d values): an exponent e and d codes in e4m3.  e is the smallest
integer in [-32, 80] with max|x| <= 448 * 2^e over the row's finite values, held as the byte e + 127; a value is
code * 2^e, the code is x * 2^-e rounded to e4m3 (nearest even, saturating).  A cache is paged ([pages, H_kv, page, d]
with a table of page ids per request) or dense ([B, H_kv, tokens, d]).
"""
import math

import numpy as np
import torch

own = False

# Most codes of K (tokens over all requests x kv-heads x d) of a drawn case: a third of the largest listed one's.
_MOST = 1 << 28


def _case(name, kind, B, H_q, H_kv, d, T_q, lo, hi, page):
    c = dict(kind=kind, B=B, H_q=H_q, H_kv=H_kv, d=d, T_q=T_q, lo=lo, hi=hi, page=page)
    if name:
        c["name"] = name
    return c


def listed():
    """For `write`, lo..hi is how many rows a request's call carries (T_q > 1: accepted rows out of T_q candidates);
    for the others, how many tokens a request has in the cache."""
    return [
        # decoding: every request's newest token joins the cache before the step's attention
        _case("write_new_tokens", "write", 16, 32, 8, 128, 1, 1, 1, 64),
        # the end of a verification round: the accepted ones of 8 candidates join the cache
        _case("write_accepted", "write", 32, 32, 8, 128, 8, 1, 8, 16),
        # prompts of a batch, written after their prefill
        _case("write_prompts", "write", 8, 32, 8, 128, 1, 9001, 16384, 64),
        # the tails of short requests go back to bf16
        _case("read_tails", "read", 8, 8, 2, 64, 1, 65, 257, 8),
        # whole histories go back to bf16 for the bf16 path
        _case("read_histories", "read", 16, 32, 8, 128, 1, 4096, 16384, 64),
        # one short request on a small model: nothing but latency
        _case("decode_tiny", "decode", 1, 4, 1, 64, 1, 1024, 1024, 16),
        # one request with a long history: a few kv-heads have to fill the GPU
        _case("decode_one_long", "decode", 1, 32, 8, 128, 1, 131071, 131071, 64),
        # a batch of equally long histories, Qwen3-8B-shaped
        _case("decode_batch", "decode", 16, 32, 8, 128, 1, 32768, 32768, 64),
        # a ragged batch in small pages
        _case("decode_ragged", "decode", 32, 32, 8, 128, 1, 8192, 65536, 16),
        # a small dense round: 4 drafts and the pending token
        _case("verify_small", "verify", 2, 8, 2, 64, 5, 700, 1531, 0),
        # the Qwen3-8B-shaped round: 8 candidates
        _case("verify_batch", "verify", 16, 32, 8, 128, 8, 32768, 32768, 128),
        # long ragged histories, 6 candidates, InternLM2.5-7B-shaped
        _case("verify_long_ragged", "verify", 8, 32, 8, 128, 6, 65536, 131072, 64),
    ]


def draw(rng):
    kind = rng.choice(["write", "read", "decode", "verify"])
    d = rng.choice([64, 128])
    H_kv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    page = rng.choice([0, 8, 16, 32, 64, 128, 256])
    T_q = rng.randint(2, 8) if kind == "verify" else 1
    if kind == "write" and rng.random() < 0.5:
        T_q = rng.randint(2, 8)
    hi = int(round(math.exp(rng.uniform(0.0, math.log(65536.0)))))
    if kind == "write" and T_q > 1:
        hi = T_q
    most_b = max(1, min(48, _MOST // (hi * H_kv * d)))
    B = int(round(math.exp(rng.uniform(0.0, math.log(most_b)))))
    lo = max(1, int(hi * rng.choice([1.0, 0.5, 0.1])))
    return _case(None, kind, B, H_kv * G, H_kv, d, T_q, lo, hi, page)


def _lengths(c):
    """Lengths of the requests: spread over lo..hi, in no order."""
    span = c["hi"] - c["lo"]
    return [c["lo"] + int(round(span * ((0.37 + b * 0.6180339887498949) % 1.0))) for b in range(c["B"])]


def _room(c):
    """Tokens that the cache holds for a request."""
    top = c["hi"] + (c["T_q"] + 64 if c["kind"] == "write" else 0)
    return -(-top // c["page"]) * c["page"] if c["page"] else -(-top // 8) * 8


def _normal(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _power(e):
    """2^e as fp32, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x):
    """fp32 rows -> (codes as float8, exponent bytes)."""
    mag = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    m, ex = torch.frexp(mag)                                   # mag = m * 2^ex, m in [0.5, 1)
    e = torch.where(m > 0.875, ex - 8, ex - 9)                 # 448 = 0.875 * 2^9
    e = torch.where(mag == 0, torch.full_like(e, -32), e).clamp(-32, 80)
    y = x * _power(-e).unsqueeze(-1)
    return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _decode(codes, scale):
    return codes.float() * _power(scale.to(torch.int32) - 127).unsqueeze(-1)


def _caches(c, gen, lens, finite):
    """Cache buffers: outer = pages in a shuffled order, or requests.  What no request holds is stale memory."""
    B, H_kv, d, page = c["B"], c["H_kv"], c["d"], c["page"]
    room = _room(c)
    per = room // page if page else 1
    outer, tokens = (B * per + 3, page) if page else (B, room)
    table = None
    if page:
        ids = torch.randperm(outer, generator=gen, device="cuda")[: B * per].to(torch.int32)
        table = ids.view(B, per)
    out = {}
    for name in ("K", "V"):
        codes = torch.empty(outer, H_kv, tokens, d, dtype=torch.uint8, device="cuda")
        scale = torch.empty(outer, H_kv, tokens, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (H_kv * tokens * d))
        for i in range(0, outer, step):
            x = _normal(gen, (min(step, outer - i), H_kv, tokens, d))
            if name == "K":
                x[..., :: d // 4] *= 4.0                       # a few channels of K stand out
            else:
                x *= torch.exp(_normal(gen, x.shape[:3]) * 0.5).unsqueeze(-1)
            q, s = _encode(x.bfloat16().float())
            codes[i:i + step], scale[i:i + step] = q.view(torch.uint8), s
        out[name], out[name + "_scale"] = codes, scale
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if not finite:                                             # behind a request's last token: anything, NaN too
        pos = torch.arange(room, device="cuda")
        dead = pos >= length.unsqueeze(1)                      # [B, room]
        b, t = dead.nonzero(as_tuple=True)
        o, i = (table[b, t // page].long(), t % page) if page else (b, t)
        for name in ("K", "V"):
            out[name][o, :, i] = 0x7F
    return out | {"table": table, "len": length}


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    lens = _lengths(c)
    B, H_q, H_kv, d, T = c["B"], c["H_q"], c["H_kv"], c["d"], c["T_q"]
    kind = c["kind"]
    s = {"case": c, "scale": d ** -0.5}
    if kind == "write":
        room = _room(c)
        s |= _caches(c, gen, [room] * B, True)
        rows = T if T > 1 else c["hi"]
        s["K_new"] = (_normal(gen, (B, H_kv, rows, d))).bfloat16()
        s["V_new"] = (_normal(gen, (B, H_kv, rows, d)) * 0.5).bfloat16()
        s["cnt"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        off = torch.tensor([(13 * b + 5) % (room - c["hi"] + 1) for b in range(B)], dtype=torch.int32, device="cuda")
        s["off"] = off
        s["idx"] = None
        if T > 1:                                              # a path through the candidates, in order
            pick = torch.rand(B, T, generator=gen, device="cuda").argsort(1)
            keep = torch.arange(T, device="cuda") < s["cnt"].unsqueeze(1)
            pick = torch.where(keep, pick, torch.full_like(pick, T)).sort(1).values
            s["idx"] = pick.clamp(max=T - 1).to(torch.int32).contiguous()
    else:
        s |= _caches(c, gen, lens, kind == "read")
        if kind == "read":
            s["off"] = torch.zeros(B, dtype=torch.int32, device="cuda")
            s["K_out"] = torch.zeros(B, H_kv, c["hi"], d, dtype=torch.bfloat16, device="cuda")
            s["V_out"] = torch.zeros_like(s["K_out"])
        else:
            u = torch.sign(_normal(gen, (H_kv, d)))            # the direction that every query shares
            q = _normal(gen, (B, H_kv, H_q // H_kv, T, d)) + 0.5 * u.view(1, H_kv, 1, 1, d)
            s["Q"] = q.reshape(B, H_q, T, d).bfloat16()
            first = (s["table"][:, 0].long() if c["page"] else torch.arange(B, device="cuda"))
            sink, e = _encode(2.0 * u)                         # the first token draws attention, its V is small
            s["K"][first, :, 0], s["K_scale"][first, :, 0] = sink.view(torch.uint8), e
            s["V_scale"][first, :, 0] -= 3
            s["O"] = torch.empty_like(s["Q"])
            s["LSE"] = torch.empty(B, H_q, T, device="cuda")
            if kind == "verify":
                s["K_loc"] = _normal(gen, (B, H_kv, T, d)).bfloat16()
                s["V_loc"] = _normal(gen, (B, H_kv, T, d)).bfloat16()
    if own:
        from paper_2609_33184_b200 import binding as ss
        s["ctx"] = ss.Context(B, H_q, H_kv, d, T, T, _room(c))
        s["cache"] = ss.Cache8(s["K"], s["V"], s["K_scale"], s["V_scale"], s["table"])
    return s


def _slots(s, tokens):
    """(outer index, token index) of tokens [B, n] of the requests, those outside taken as 0."""
    B = tokens.shape[0]
    if s["table"] is None:
        return torch.arange(B, device="cuda").unsqueeze(1).expand_as(tokens), tokens
    page = s["case"]["page"]
    return torch.gather(s["table"].long(), 1, tokens // page), tokens % page


def _rows(s, name, n):
    """The first n tokens of every request as fp32 [B, H_kv, n, d]."""
    tokens = torch.arange(n, device="cuda").unsqueeze(0).expand(s["case"]["B"], n)
    o, i = _slots(s, tokens)
    x = _decode(s[name][o, :, i].view(torch.float8_e4m3fn), s[name + "_scale"][o, :, i])   # [B, n, H_kv, d]
    return x.transpose(1, 2)


def _plain_write(s):
    rows = s["K_new"].shape[2]
    k = torch.arange(rows, device="cuda")
    b, k = (k.unsqueeze(0) < s["cnt"].unsqueeze(1)).nonzero(as_tuple=True)
    src = k if s["idx"] is None else s["idx"].long()[b, k]
    tok = s["off"].long()[b] + k
    page = s["case"]["page"]
    o, i = (s["table"].long()[b, tok // page], tok % page) if page else (b, tok)
    for name in ("K", "V"):
        q, e = _encode(s[name + "_new"][b, :, src].float())
        s[name][o, :, i], s[name + "_scale"][o, :, i] = q.view(torch.uint8), e


def _plain_read(s):
    n = s["case"]["hi"]
    live = (torch.arange(n, device="cuda").unsqueeze(0) < s["len"].unsqueeze(1)).view(-1, 1, n, 1)
    return tuple(torch.where(live, _rows(s, name, n).bfloat16(), s[name + "_out"]) for name in ("K", "V"))


def _plain_attention(s):
    c = s["case"]
    B, H_q, H_kv, d, T = c["B"], c["H_q"], c["H_kv"], c["d"], c["T_q"]
    n = c["hi"]
    q = s["Q"].float().reshape(B, H_kv, -1, d) * s["scale"]
    live = (torch.arange(n, device="cuda").unsqueeze(0) < s["len"].unsqueeze(1)).view(B, 1, 1, n)
    score = torch.where(live, q @ _rows(s, "K", n).transpose(2, 3), torch.full((), -math.inf, device="cuda"))
    top = score.amax(-1, keepdim=True)
    if c["kind"] == "verify":
        i = torch.arange(T, device="cuda").repeat(H_q // H_kv)
        seen = torch.arange(T, device="cuda").unsqueeze(0) <= i.unsqueeze(1)
        near = q @ s["K_loc"].float().transpose(2, 3)
        near = torch.where(seen, near, torch.full((), -math.inf, device="cuda"))
        top = torch.maximum(top, near.amax(-1, keepdim=True))
    w = torch.exp(score - top)
    V = torch.where(live.transpose(2, 3), _rows(s, "V", n), torch.zeros((), device="cuda"))
    total, out = w.sum(-1, keepdim=True), w @ V
    if c["kind"] == "verify":
        w = torch.exp(near - top)
        total, out = total + w.sum(-1, keepdim=True), out + w @ s["V_loc"].float()
    lse = (top + torch.log(total)).reshape(B, H_q, T)
    return (out / total).reshape(B, H_q, T, d).bfloat16(), lse


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        ctx, cache = s["ctx"], s["cache"]
        if kind == "write":
            ctx.ss_kv8_write(cache, s["K_new"], s["V_new"], s["off"], s["cnt"], s["idx"])
        elif kind == "read":
            ctx.ss_kv8_read(cache, s["K_out"], s["V_out"], s["off"], s["len"])
            return s["K_out"], s["V_out"]
        elif kind == "decode":
            ctx.ss_decode8(s["Q"], s["scale"], cache, s["len"], s["O"], s["LSE"])
            return s["O"], s["LSE"]
        else:
            ctx.ss_verify_begin(s["Q"], s["scale"])
            ctx.ss_verify_chunk8(cache, s["len"])
            ctx.ss_verify_local(s["K_loc"], s["V_loc"])
            ctx.ss_verify_finalize(s["O"], s["LSE"])
            return s["O"], s["LSE"]
    elif kind == "write":
        _plain_write(s)
    else:
        return _plain_read(s) if kind == "read" else _plain_attention(s)
    # the whole cache: the codes' values and the rows' exponents
    f8 = torch.float8_e4m3fn
    return s["K"].view(f8), s["K_scale"], s["V"].view(f8), s["V_scale"]


def work(case):
    c = case
    n, d, H_kv = sum(_lengths(c)), c["d"], c["H_kv"]
    rows = c["B"] * c["H_q"] * c["T_q"]
    if c["kind"] in ("write", "read"):                         # bf16 rows one way, codes and exponents the other
        return {"bytes": n * H_kv * 2 * (3 * d + 1), "flops": n * H_kv * 2 * 2 * d}
    R = c["H_q"] // H_kv * c["T_q"]
    byte, flop = n * H_kv * 2 * (d + 1) + rows * (4 * d + 4), 4 * n * H_kv * R * d
    if c["kind"] == "verify":
        byte += c["B"] * H_kv * c["T_q"] * 4 * d
        flop += 2 * rows * (c["T_q"] + 1) * d
    return {"bytes": byte, "flops": flop}


def _exact_code(x):
    """A row's values in 64 bits -> (the e4m3 values of its codes, its exponent byte), from the format's definition."""
    mag = np.abs(x)
    top = np.where(np.isfinite(mag), mag, 0.0).max(-1)
    e = np.full(top.shape, -32, dtype=np.int64)
    some = top > 0
    e[some] = np.clip(np.ceil(np.log2(top[some] / 448.0) - 1e-13), -32, 80).astype(np.int64)
    e += (top > 448.0 * np.exp2(e.astype(np.float64))) & (e < 80)
    y = np.clip(x * np.exp2(-e.astype(np.float64))[..., None], -448.0, 448.0)
    grain = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 1e-300))), -6.0) - 3.0)
    return np.rint(y / grain) * grain, (e + 127).astype(np.uint8)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind, B, H_kv, d, T = c["kind"], c["B"], c["H_kv"], c["d"], c["T_q"]
    lens, page = _lengths(c), c["page"]
    if sum(lens) * H_kv * d > (1 << 25) and kind == "write":
        return None
    if kind == "write":
        out = {}
        for name in ("K", "V"):
            codes = s[name].view(torch.float8_e4m3fn).double().cpu().numpy()
            scale = s[name + "_scale"].cpu().numpy()
            new = s[name + "_new"].double().cpu().numpy()
            for b in range(B):
                for k in range(lens[b]):
                    j = k if s["idx"] is None else int(s["idx"][b, k])
                    t = int(s["off"][b]) + k
                    o, i = (int(s["table"][b, t // page]), t % page) if page else (b, t)
                    codes[o, :, i], scale[o, :, i] = _exact_code(new[b, :, j])
            out[name] = (codes, scale)
        return out["K"][0], out["K"][1], out["V"][0], out["V"][1]

    # from here in 64 bits on the device, one request at a time
    def history(name, b, n):
        if page:
            pages = s["table"][b, : -(-n // page)].long()
            q, e = s[name][pages], s[name + "_scale"][pages]
            q, e = q.transpose(0, 1).reshape(H_kv, -1, d), e.transpose(0, 1).reshape(H_kv, -1)
        else:
            q, e = s[name][b], s[name + "_scale"][b]
        q, e = q[:, :n].to(torch.int16), e[:, :n].double()
        field, frac = (q >> 3) & 15, (q & 7).double()
        val = torch.where(field == 0, frac * 2.0 ** -9, (1.0 + frac / 8.0) * torch.exp2(field.double() - 7.0))
        return torch.where(q >= 128, -val, val) * torch.exp2(e - 127.0).unsqueeze(-1)

    if kind == "read":
        K = torch.zeros(B, H_kv, c["hi"], d, dtype=torch.float64)
        V = torch.zeros_like(K)
        for b, n in enumerate(lens):
            K[b, :, :n], V[b, :, :n] = history("K", b, n).cpu(), history("V", b, n).cpu()
        return K, V
    G = c["H_q"] // H_kv
    O = torch.zeros(B, H_kv, G, T, d, dtype=torch.float64)
    L = torch.zeros(B, H_kv, G, T, dtype=torch.float64)
    for b, n in enumerate(lens):
        K, V = history("K", b, n), history("V", b, n)
        for h in range(H_kv):
            q = s["Q"][b, h * G:(h + 1) * G].double()          # [G, T, d]
            a = torch.einsum("gtd,nd->gtn", q, K[h]) * s["scale"]
            v = V[h]
            if kind == "verify":
                near = torch.einsum("gtd,nd->gtn", q, s["K_loc"][b, h].double()) * s["scale"]
                near = near.masked_fill(torch.ones(T, T, device="cuda").triu(1).bool(), -math.inf)
                a, v = torch.cat([a, near], -1), torch.cat([v, s["V_loc"][b, h].double()])
            L[b, h] = torch.logsumexp(a, -1).cpu()
            O[b, h] = torch.einsum("gtn,nd->gtd", torch.softmax(a, -1), v).cpu()
    return O.reshape(B, c["H_q"], T, d), L.reshape(B, c["H_q"], T)
