"""Cases of the 8-bit paged KV cache and of the rotary positions with several axes.

Four operators, the steps of one layer that writes its keys and values into an 8-bit cache
and attends over it:

  rope    rotary positions with several axes (time, height, width) applied to the query and
          key rows of a step, forward and inverse (the inverse is the gradient, and takes a
          rotation off again)
  append  the step's key and value rows written into pages of 8-bit floating point (e4m3)
          with one power-of-two scale for each page and KV head
  read    rows of the cache back in 16 or 32 bits
  attend  the step's query rows over their requests' pages, from one row a request to chunks
          of a prompt

`run` computes them by elementary torch operations where `own` is false and by the
framework's entry points where it is true.  `exact` computes them from their definitions in
64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA = 1000000.0
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------
# cases

def listed():
    """Shapes: 28 query and 4 KV heads or 64 and 8 at 128 dimensions, 8 and 4 at 64."""
    return [
        # one token of each of 16 requests: what a decode step rotates in one layer
        dict(name="rope step", kind="rope", rows=16, Hq=28, Hkv=4, d=128, dtype="bf16", order="sectioned",
             pairing="halves", inverse=False),
        # an odd number of rows in 32 bits, the rotation taken off (the gradient)
        dict(name="rope back f32", kind="rope", rows=1023, Hq=8, Hkv=4, d=64, dtype="f32", order="interleaved",
             pairing="adjacent", inverse=True),
        # the prompt of a long video on the wide shape
        dict(name="rope video", kind="rope", rows=32768, Hq=64, Hkv=8, d=128, dtype="bf16", order="interleaved",
             pairing="halves", inverse=False),
        # a decode step writes one row of each of 64 requests into partly filled pages
        dict(name="append step", kind="append", requests=64, rows=1, context=12544, Hkv=4, d=128, page=64,
             dtype="bf16"),
        # short ragged prompts in 32 bits, small pages, ends inside a page
        dict(name="append prompts f32", kind="append", requests=7, rows=777, context=100, Hkv=4, d=64, page=16,
             dtype="f32"),
        # the visual tokens of a long video
        dict(name="append video", kind="append", requests=1, rows=32768, context=0, Hkv=8, d=128, page=64,
             dtype="bf16"),
        # a short cache back in 32 bits
        dict(name="read short f32", kind="read", requests=3, context=333, Hkv=4, d=64, page=16, dtype="f32"),
        # a batch of video caches back in 16 bits
        dict(name="read batch", kind="read", requests=16, context=12544, Hkv=4, d=128, page=64, dtype="bf16"),
        # one request's next token over a short cache: latency
        dict(name="attend step short", kind="attend", requests=1, rows=1, context=777, Hq=28, Hkv=4, d=128,
             page=64, dtype="bf16", causal=True),
        # a batch's next tokens over long ragged caches: the cache's bytes
        dict(name="attend step batch", kind="attend", requests=32, rows=1, context=32768, Hq=64, Hkv=8, d=128,
             page=64, dtype="bf16", causal=True),
        # a few rows a request (drafted tokens) in 32 bits
        dict(name="attend drafts f32", kind="attend", requests=6, rows=5, context=3136, Hq=8, Hkv=4, d=64,
             page=16, dtype="f32", causal=True),
        # a chunk of a long prompt over what came before it: the products
        dict(name="attend chunk", kind="attend", requests=1, rows=2048, context=32768, Hq=64, Hkv=8, d=128,
             page=64, dtype="bf16", causal=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "read", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Hq, Hkv, d = rng.choice([(28, 4, 128), (64, 8, 128), (8, 4, 64), (8, 8, 128), (16, 1, 64)])
    page = rng.choice([16, 32, 64, 128])
    if kind == "rope":
        most = 32768 * 72 * 128 * 2 // ((Hq + Hkv) * d * (2 if dtype == "bf16" else 4))
        return dict(kind=kind, rows=_log_int(rng, 1, min(most, 32768)), Hq=Hq, Hkv=Hkv, d=d, dtype=dtype,
                    order=rng.choice(["sectioned", "interleaved"]), pairing=rng.choice(["halves", "adjacent"]),
                    inverse=rng.random() < 0.5)
    if kind == "append":
        n = _log_int(rng, 1, 64)
        most = 32768 * 8 * 128 * 2 // (n * Hkv * d * (2 if dtype == "bf16" else 4))
        return dict(kind=kind, requests=n, rows=_log_int(rng, 1, max(1, min(most, 32768))),
                    context=rng.choice([0, _log_int(rng, 1, 4096)]), Hkv=Hkv, d=d, page=page, dtype=dtype)
    if kind == "read":
        n = _log_int(rng, 1, 64)
        most = 16 * 12544 * 4 * 128 * 2 // (n * Hkv * d * (2 if dtype == "bf16" else 4))
        return dict(kind=kind, requests=n, context=_log_int(rng, 1, max(1, min(most, 32768))), Hkv=Hkv, d=d,
                    page=page, dtype=dtype)
    causal = rng.random() < 0.8
    if rng.random() < 0.6:      # one or a few rows a request
        n, rows = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 7])
        most = 32 * 32768 * 8 * 128 // (n * Hkv * d)
    else:                       # chunks of prompts
        n, rows = _log_int(rng, 1, 8), _log_int(rng, 8, 2048)
        most = 2048 * 32768 * 64 * 128 // (n * rows * Hq * d * (8 if dtype == "f32" else 1))
    context = _log_int(rng, 1, max(1, min(most, 32768)))
    return dict(kind=kind, requests=n, rows=min(rows, context) if causal else rows, context=context, Hq=Hq,
                Hkv=Hkv, d=d, page=page, dtype=dtype, causal=causal)


def _rows(c):
    """New rows of each request: the case's for the first, fewer for the later ones."""
    n, m = c["requests"], c["rows"]
    return [max(1, m - r * m // (2 * n)) for r in range(n)]


def _lens(c):
    """Tokens in the cache of each request, the step's rows included: from the case's number
    down to a quarter of it; in batches of four and more the last request is empty (a padding
    entry), so an attention row there sees nothing."""
    n, top = c["requests"], c["context"]
    if c["kind"] == "append":
        return [m + max(0, top - r * top * 3 // (4 * n)) for r, m in enumerate(_rows(c))]
    lens = [max(1, top - r * top * 3 // (4 * n)) for r in range(n)]
    if c["kind"] == "attend":
        lens = [max(x, m) for x, m in zip(lens, _rows(c))]
    if n >= 4:
        lens[-1] = 0
    return lens


def _sections(c):
    return [c["d"] // 8, 3 * c["d"] // 16, 3 * c["d"] // 16]


def work(case):
    c = case
    size = 2 if c.get("dtype") == "bf16" else 4
    if c["kind"] == "rope":
        n = c["rows"] * (c["Hq"] + c["Hkv"]) * c["d"]
        return {"bytes": 2 * n * size + 12 * c["rows"], "flops": 3 * n}
    lens = _lens(c)
    pages = sum(-(-x // c["page"]) for x in lens)
    row = c["Hkv"] * c["d"]
    if c["kind"] == "append":
        m = _rows(c)
        touched = sum(-(-x // c["page"]) - (x - k) // c["page"] for x, k in zip(lens, m))
        return {"bytes": 2 * sum(m) * row * (size + 1) + touched * (4 + 8 * c["Hkv"]), "flops": 4 * sum(m) * row}
    if c["kind"] == "read":
        return {"bytes": 2 * sum(lens) * row * (size + 1) + pages * (4 + 8 * c["Hkv"]), "flops": 2 * sum(lens) * row}
    m = _rows(c)
    seen = 0
    for x, k in zip(lens, m):
        k = min(k, x)
        seen += k * x - k * (k - 1) // 2 if c["causal"] else k * x
    return {"bytes": 2 * sum(lens) * row + pages * (4 + 8 * c["Hkv"]) + 2 * sum(m) * c["Hq"] * c["d"] * size
            + 4 * sum(m) * c["Hq"], "flops": 4 * seen * c["Hq"] * c["d"]}


# ---------------------------------------------------------------------------------------
# inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g)


def _scale_of(amax):
    """The least power of two 2^e, e >= -126, with amax <= 448 * 2^e; 0 for amax 0."""
    m, k = torch.frexp(amax)
    e = torch.where(m <= 0.875, k - 9, k - 8).clamp(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.zeros_like(amax))


def _encode(x, scale):
    """e4m3 codes (uint8) of x / scale, to nearest even; what is not finite becomes NaN."""
    s = torch.where(scale > 0, scale, torch.ones_like(scale))
    y = torch.where(torch.isfinite(x), x / s, torch.full_like(x, float("nan")))
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes, scale):
    return codes.view(torch.float8_e4m3fn).to(torch.float32) * scale


def _video_positions(rows):
    """(time, height, width) of each row: frames of 14 x 14 tokens, then text on one axis."""
    i = torch.arange(rows, device=DEV)
    vis = rows * 7 // 8
    t, h, w = i // 196, i % 196 // 14, i % 14
    last = (vis + 195) // 196
    text = last + (i - vis)
    return torch.stack([torch.where(i < vis, x, text) for x in (t, h, w)]).to(torch.int32).contiguous()


def _pool(c, g, lens, filled):
    """A paged cache whose requests hold `filled` tokens each: codes, scales, block table.
    Keys have a few channels ten times as wide, the first token is a sink with small values.
    Slots that no token was written to hold what was there before (NaN codes among it) where
    nothing returns them."""
    n, page, Hkv, d = c["requests"], c["page"], c["Hkv"], c["d"]
    need = [-(-x // page) for x in lens]
    width = max(1, max(need))
    n_pages = sum(need) + 3
    table = torch.zeros((n, width), dtype=torch.int64, device=DEV)
    order = torch.randperm(n_pages - 1, generator=g, device=DEV) + 1       # page 0 is no one's
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = order[at:at + k]
        at += k
    have = torch.zeros(n_pages, dtype=torch.int64, device=DEV)            # tokens in each page
    for r, x in enumerate(filled):
        k = -(-x // page)
        if k:
            have[table[r, :k]] = page
            have[table[r, k - 1]] = x - (k - 1) * page
    live = (torch.arange(page, device=DEV) < have[:, None])[:, None, :, None]
    out = []
    for kind in range(2):
        x = _normal(g, n_pages, Hkv, page, d)
        if kind == 0:
            x[..., ::50] *= 10.0
        else:
            for r, k in enumerate(need):
                if k:
                    x[table[r, 0], :, 0] *= 0.01
        x *= live
        scale = _scale_of(x.abs().amax(dim=(2, 3)))
        codes = _encode(x, scale[:, :, None, None])
        if c["kind"] != "append":
            codes = torch.where(live, codes, torch.full_like(codes, 0x7F))
        out += [codes, scale]
        del x
    return out[0], out[1], out[2], out[3], table.to(torch.int32)


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = TYPES[c["dtype"]]
    s = dict(case=dict(case))
    if c["kind"] == "rope":
        # the fused projection's output: a row holds its query, key and value heads
        qkv = _normal(g, c["rows"], c["Hq"] + 2 * c["Hkv"], c["d"]).to(dt)
        start = torch.randint(0, 1000, (1,), generator=g, device=DEV, dtype=torch.int32)
        s.update(qkv=qkv, positions=_video_positions(c["rows"]) + start,
                 q_out=torch.empty((c["rows"], c["Hq"], c["d"]), dtype=dt, device=DEV),
                 k_out=torch.empty((c["rows"], c["Hkv"], c["d"]), dtype=dt, device=DEV))
        if own:
            from paper_2608_24063_gb300 import viscache as vc
            s["rope"] = vc.make_rope(_sections(c), THETA, interleaved=c["order"] == "interleaved",
                                     adjacent=c["pairing"] == "adjacent")
        return s
    lens = _lens(c)
    rows = lens if c["kind"] == "read" else _rows(c)
    filled = [x - m for x, m in zip(lens, rows)] if c["kind"] == "append" else lens
    kc, ks, vc_, vs, table = _pool(c, g, lens, filled)
    start = [0]
    for m in rows:
        start.append(start[-1] + m)
    total = start[-1]
    s.update(K_codes=kc, K_scale=ks, V_codes=vc_, V_scale=vs, table=table, rows=total,
             seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
             row_start=torch.tensor(start, dtype=torch.int32, device=DEV))
    if c["kind"] == "append":
        kv = _normal(g, total, 2 * c["Hkv"], c["d"])
        kv[:, :c["Hkv"], ::50] *= 10.0
        s["kv"] = kv.to(dt)
    elif c["kind"] == "read":
        s["K_hat"] = torch.empty((total, c["Hkv"], c["d"]), dtype=dt, device=DEV)
        s["V_hat"] = torch.empty((total, c["Hkv"], c["d"]), dtype=dt, device=DEV)
    else:
        s["q"] = (_normal(g, total, c["Hq"], c["d"]) * 1.5).to(dt)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((total, c["Hq"]), dtype=torch.float32, device=DEV)
    if own:
        from paper_2608_24063_gb300 import viscache as vc
        s["cache"] = vc.Kv8Cache(kc, vc_, ks, vs)
        s["step"] = vc.Kv8Step(table, s["seq_lens"], s["row_start"], total)
        s["ws"] = torch.empty(vc.viscache_kv8_workspace_size(total, c.get("Hq", c["Hkv"]), c["Hkv"], c["d"]),
                              dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------------------
# one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"rope": _plain_rope, "append": _plain_append, "read": _plain_read, "attend": _plain_attend}[kind](state)


def _own(kind, s):
    from paper_2608_24063_gb300 import viscache as vc
    c = s["case"]
    if kind == "rope":
        q, k = s["qkv"][:, :c["Hq"]], s["qkv"][:, c["Hq"]:c["Hq"] + c["Hkv"]]
        vc.viscache_mrope(s["rope"], s["positions"], q, k, inverse=c["inverse"], q_out=s["q_out"], k_out=s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "append":
        k, v = s["kv"][:, :c["Hkv"]], s["kv"][:, c["Hkv"]:]
        vc.viscache_kv8_append(s["cache"], s["step"], k, v, ws=s["ws"])
        return _pool_values(s)
    if kind == "read":
        vc.viscache_kv8_read(s["cache"], s["step"], out=(s["K_hat"], s["V_hat"]), ws=s["ws"])
        return {"K": s["K_hat"], "V": s["V_hat"]}
    vc.viscache_kv8_attention(s["cache"], s["step"], s["q"], causal=c["causal"], out=s["out"], lse=s["lse"],
                              ws=s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _pool_values(s):
    """The cache's codes as the 8-bit numbers they are, and their scales."""
    return {"K": s["K_codes"].view(torch.float8_e4m3fn), "K_scale": s["K_scale"],
            "V": s["V_codes"].view(torch.float8_e4m3fn), "V_scale": s["V_scale"]}


def _axis_of(c):
    """The axis whose position turns frequency i of d / 2."""
    sec, half = _sections(c), c["d"] // 2
    i = torch.arange(half, device=DEV)
    if c["order"] == "interleaved":     # i mod 3 while that axis has frequencies left, axis 0 after
        a = i % 3
        return torch.where(i < 3 * torch.tensor(sec, device=DEV)[a], a, torch.zeros_like(a))
    return (i >= sec[0]).long() + (i >= sec[0] + sec[1]).long()


def _plain_rope(s):
    c = s["case"]
    d, half = c["d"], c["d"] // 2
    # phase in turns as a 40-bit fraction, so that large positions keep their digits in 32 bits
    i = torch.arange(half, dtype=torch.float64, device=DEV)
    f = (THETA ** (-i / half) / (2 * math.pi) * 2.0 ** 40).round().to(torch.int64)
    p = s["positions"].to(torch.int64)[_axis_of(c)].t()                     # [rows][half]
    angle = ((p * f) & ((1 << 40) - 1)).to(torch.float32) * (2 * math.pi / 2.0 ** 40)
    cos, sin = angle.cos()[:, None, :], angle.sin()[:, None, :]
    if c["inverse"]:
        sin = -sin
    x = s["qkv"][:, :c["Hq"] + c["Hkv"]].float()
    if c["pairing"] == "halves":
        a, b = x[..., :half], x[..., half:]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0::2], x[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    y = y.to(s["qkv"].dtype)
    return {"q": y[:, :c["Hq"]], "k": y[:, c["Hq"]:]}


def _plain_append(s):
    c = s["case"]
    page = c["page"]
    lens, start = s["seq_lens"].long(), s["row_start"].long()
    old = lens - (start[1:] - start[:-1])
    first = old // page
    most = max(-(-x // page) - (x - m) // page for x, m in zip(_lens(c), _rows(c)))
    j = first[:, None] + torch.arange(most, device=DEV)                     # [n][pages]
    used = j * page < lens[:, None]
    pid = torch.where(used, s["table"].long().gather(1, j.clamp(max=s["table"].shape[1] - 1)), torch.zeros_like(j))
    pos = j[:, :, None] * page + torch.arange(page, device=DEV)             # [n][pages][slots]
    new = (pos >= old[:, None, None]) & (pos < lens[:, None, None])
    kept = (pos < old[:, None, None]) & used[:, :, None]
    row = (start[:-1, None, None] + pos - old[:, None, None]).clamp(0, s["rows"] - 1)
    new, kept = new[:, :, None, :, None], kept[:, :, None, :, None]
    for x, codes, scale in ((s["kv"][:, :c["Hkv"]], s["K_codes"], s["K_scale"]),
                            (s["kv"][:, c["Hkv"]:], s["V_codes"], s["V_scale"])):
        y = x[row].float().transpose(2, 3)                                  # [n][pages][Hkv][slots][d]
        good = new & torch.isfinite(y)
        amax = torch.where(good, y.abs(), torch.zeros_like(y)).amax(dim=(3, 4))
        was = torch.where(kept.any(dim=3)[..., 0], scale[pid], torch.zeros_like(amax))
        now = torch.maximum(was, _scale_of(amax))
        there = codes[pid]
        c_old = _encode(_decode(there, was[..., None, None]), now[..., None, None])
        c_new = _encode(y, now[..., None, None])
        out = torch.where(new, c_new, torch.where(kept, c_old, there))
        codes[pid] = out
        scale[pid] = torch.where(used[..., None], now, scale[pid])
    return _pool_values(s)


def _gathered(s, c):
    """Values [n][Hkv][slots][d] in 32 bits of every request's pages."""
    t = s["table"].long()
    return [(_decode(codes[t], scale[t][..., None, None]).transpose(1, 2).flatten(2, 3))
            for codes, scale in ((s["K_codes"], s["K_scale"]), (s["V_codes"], s["V_scale"]))]


def _plain_read(s):
    c = s["case"]
    start = s["row_start"].long()
    i = torch.arange(s["rows"], device=DEV)
    r = torch.searchsorted(start, i, right=True) - 1
    at = i - start[r] + s["seq_lens"].long()[r] - (start[r + 1] - start[r])
    page, slot = s["table"].long()[r, at // c["page"]], at % c["page"]
    K, V = (_decode(codes[page, :, slot], scale[page][..., None]).to(TYPES[c["dtype"]])
            for codes, scale in ((s["K_codes"], s["K_scale"]), (s["V_codes"], s["V_scale"])))
    return {"K": K, "V": V}


def _plain_attend(s):
    c = s["case"]
    n, Hq, Hkv, d, G = c["requests"], c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    start, lens = s["row_start"].long(), s["seq_lens"].long()
    m = max(_rows(c))
    i = torch.arange(m, device=DEV)
    count = start[1:] - start[:-1]
    there = i < count[:, None]                                             # [n][m]
    row = (start[:-1, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"][row].float().view(n, m, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, m * G, d)
    K, V = _gathered(s, c)
    slots = K.shape[2]
    t = torch.arange(slots, device=DEV)
    live = (t < lens[:, None])[:, None, :]                                 # [n][1][slots]
    V = torch.where(live[..., None], V, torch.zeros_like(V))
    x = torch.matmul(q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    del K
    seen = live.expand(n, m, slots)
    if c["causal"]:
        seen = seen & (t <= (lens - count)[:, None, None] + i[:, None])
    seen = seen[:, None, :, None, :].expand(n, 1, m, G, slots).reshape(n, 1, m * G, slots)
    x.masked_fill_(~seen, float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = x.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p, V) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log()).view(n, Hkv, m, G).permute(0, 2, 1, 3).reshape(n, m, Hq)
    out = out.view(n, Hkv, m, G, d).permute(0, 2, 1, 3, 4).reshape(n, m, Hq, d)
    return {"out": out[there].to(TYPES[c["dtype"]]), "lse": lse[there]}


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits

def _e4m3_table():
    """Value of each of the 256 codes: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7F NaN."""
    v = []
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = math.nan if b & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v.append(-x if b & 128 else x)
    return torch.tensor(v, dtype=torch.float64, device=DEV)


def _round_e4m3(x):
    """x (64 bits, |x| <= 448) rounded to the nearest e4m3 number, ties to even."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    q = torch.exp2(e - 3)
    return torch.round(x / q) * q


def exact(case, seed):
    c = case
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64 = torch.float64
    if c["kind"] == "rope":
        half, sec = c["d"] // 2, _sections(c)
        x = s["qkv"][:, :c["Hq"] + c["Hkv"]].to(f64)
        y = torch.empty_like(x)
        for i in range(half):
            if c["order"] == "interleaved":
                a = i % 3 if i < 3 * sec[i % 3] else 0
            else:
                a = 0 if i < sec[0] else 1 if i < sec[0] + sec[1] else 2
            w = s["positions"][a].to(f64) * (THETA ** (-i / half)) * (-1.0 if c["inverse"] else 1.0)
            co, si = torch.cos(w)[:, None], torch.sin(w)[:, None]
            u, v = (i, i + half) if c["pairing"] == "halves" else (2 * i, 2 * i + 1)
            y[..., u] = x[..., u] * co - x[..., v] * si
            y[..., v] = x[..., u] * si + x[..., v] * co
        return {"q": y[:, :c["Hq"]], "k": y[:, c["Hq"]:]}
    value = _e4m3_table()
    table = s["table"].cpu().tolist()
    lens, rows, page = _lens(c), _rows(c) if c["kind"] != "read" else _lens(c), c["page"]
    if c["kind"] == "append":
        out = {}
        for name, x in (("K", s["kv"][:, :c["Hkv"]]), ("V", s["kv"][:, c["Hkv"]:])):
            codes, scale = s[name + "_codes"], s[name + "_scale"].to(f64)
            if c["requests"] > 8 and c["rows"] > 1000:
                return None
            held = value[codes.long()]
            at = 0
            for r in range(c["requests"]):
                old = lens[r] - rows[r]
                for j in range(old // page, -(-lens[r] // page)):
                    lo, hi = max(old, j * page), min(lens[r], (j + 1) * page)
                    y = x[at + lo - old:at + hi - old].to(f64).transpose(0, 1)   # [Hkv][k][d]
                    p = table[r][j]
                    amax = y.abs().amax(dim=(1, 2))
                    new = torch.exp2(torch.ceil(torch.log2(amax / 448.0)).clamp(min=-126))
                    prev = scale[p] if lo > j * page else torch.zeros_like(new)
                    now = torch.maximum(prev, new)
                    a = lo - j * page
                    if a > 0:
                        held[p, :, :a] = _round_e4m3(held[p, :, :a] * (prev / now)[:, None, None])
                    held[p, :, a:a + hi - lo] = _round_e4m3(y / now[:, None, None])
                    scale[p] = now
                at += rows[r]
            out[name], out[name + "_scale"] = held, scale
        return out
    K, V = (value[s[n + "_codes"].long()] * s[n + "_scale"].to(f64)[..., None, None]
            if c["kind"] == "read" else None for n in ("K", "V"))
    if c["kind"] == "read":
        out = {"K": [], "V": []}
        for name, x in (("K", K), ("V", V)):
            for r, length in enumerate(lens):
                k = -(-length // page)
                y = x[s["table"][r, :k].long()].transpose(1, 2).reshape(k * page, c["Hkv"], c["d"])
                out[name].append(y[:length])
            out[name] = torch.cat(out[name])
        return out
    Hq, Hkv, d, G = c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    out = torch.zeros((s["rows"], Hq, d), dtype=f64, device=DEV)
    lse = torch.full((s["rows"], Hq), -math.inf, dtype=f64, device=DEV)
    at = 0
    for r, (length, m) in enumerate(zip(lens, rows)):
        ids = s["table"][r, :-(-length // page)].long()
        for g in range(Hkv if length else 0):
            k, v = ((value[s[n + "_codes"][ids, g].long()] * s[n + "_scale"][ids, g].to(f64)[:, None, None])
                    .reshape(-1, d)[:length] for n in ("K", "V"))
            for h in range(g * G, (g + 1) * G):
                x = s["q"][at:at + m, h].to(f64) @ k.T / math.sqrt(d)
                if c["causal"]:
                    last = length - m + torch.arange(m, device=DEV)
                    x = torch.where(torch.arange(length, device=DEV) <= last[:, None], x, -math.inf)
                z = torch.logsumexp(x, dim=1)
                lse[at:at + m, h] = z
                some = torch.isfinite(z)[:, None]
                out[at:at + m, h] = torch.where(some, torch.exp(x - torch.where(some, z[:, None], 0.0)), 0.0) @ v
        at += m
    return {"out": out, "lse": lse}
