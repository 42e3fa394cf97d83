"""Cases of the operators around a decode step that keep a cache within a budget and pick the next token.

Five operators, beside the steps of a layer that writes into and attends over an 8-bit paged cache:

  turn    queries and keys normed for each head (root mean square, a weight a channel) and given
          their rotary positions with several axes in the same pass
  back    its gradient: of the rows, and of the norms' weights
  weigh   the attention probabilities of a step's rows added up for each token and KV head
  evict   the tokens with the least accumulated weight taken out of the pages of each KV head, the
          gaps closed in place
  sample  the next token of each row of logits by temperature, top-k, top-p and min-p, from given
          random numbers

`run` computes them by elementary torch operations where `own` is false and by the framework's
entry points where it is true.  `exact` computes them from their definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA = 1000000.0
EPS = 1e-6


# ---------------------------------------------------------------------------------------
# cases

def listed():
    """Shapes: 28 query and 4 KV heads or 64 and 8 at 128 dimensions, 8 and 4 at 64."""
    return [
        # one token of each of 16 requests: what a decode step norms and rotates in one layer
        dict(name="turn step", kind="turn", rows=16, Hq=28, Hkv=4, d=128, dtype="bf16", order="sectioned",
             pairing="halves"),
        # the prompt of a long video on the wide shape
        dict(name="turn video", kind="turn", rows=32768, Hq=64, Hkv=8, d=128, dtype="bf16", order="interleaved",
             pairing="halves"),
        # the gradient of an odd number of rows in 32 bits
        dict(name="back f32", kind="back", rows=1023, Hq=8, Hkv=4, d=64, dtype="f32", order="interleaved",
             pairing="adjacent"),
        # the gradient of a training step's rows
        dict(name="back train", kind="back", rows=12544, Hq=28, Hkv=4, d=128, dtype="bf16", order="sectioned",
             pairing="halves"),
        # a few rows a request (drafted tokens) in 32 bits, small pages: latency
        dict(name="weigh drafts f32", kind="weigh", requests=6, rows=5, context=3136, Hq=8, Hkv=4, d=64, page=16,
             dtype="f32", causal=True),
        # a batch's next tokens over long ragged caches: the key codes' bytes
        dict(name="weigh step batch", kind="weigh", requests=32, rows=1, context=32768, Hq=64, Hkv=8, d=128, page=64,
             dtype="bf16", causal=True),
        # a chunk of a long prompt over what came before it: products and exponentials
        dict(name="weigh chunk", kind="weigh", requests=1, rows=2048, context=32768, Hq=64, Hkv=8, d=128, page=64,
             dtype="bf16", causal=True),
        # a decode batch a page over its budget
        dict(name="evict page", kind="evict", requests=16, context=1088, keep=1024, sink=4, recent=128, Hkv=4, d=128,
             page=64),
        # ragged caches of videos cut to a quarter
        dict(name="evict videos", kind="evict", requests=16, context=12544, keep=3136, sink=4, recent=256, Hkv=8, d=128,
             page=64),
        # one request's next token, all filters on: latency
        dict(name="sample one", kind="sample", rows=1, vocab=32000, dtype="f32", filters="all"),
        # a batch without filters, an odd vocabulary
        dict(name="sample open", kind="sample", rows=64, vocab=50001, dtype="f32", filters="none"),
        # a large batch over a large vocabulary in 16 bits, rows with filters of their own
        dict(name="sample batch", kind="sample", rows=256, vocab=131072, dtype="bf16", filters="mixed"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["turn", "back", "weigh", "weigh", "evict", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Hq, Hkv, d = rng.choice([(28, 4, 128), (64, 8, 128), (8, 4, 64), (8, 8, 128), (16, 1, 64)])
    page = rng.choice([16, 32, 64, 128])
    size = 2 if dtype == "bf16" else 4
    if kind in ("turn", "back"):
        most = (32768 * 72 * 2 if kind == "turn" else 12544 * 32 * 2) * 128 // ((Hq + Hkv) * d * size)
        return dict(kind=kind, rows=_log_int(rng, 1, min(most, 32768)), Hq=Hq, Hkv=Hkv, d=d, dtype=dtype,
                    order=rng.choice(["sectioned", "interleaved"]), pairing=rng.choice(["halves", "adjacent"]))
    if kind == "weigh":
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
    if kind == "evict":
        n = _log_int(rng, 1, 64)
        context = _log_int(rng, 2, min(32768, 16 * 12544 * 8 * 128 // (n * Hkv * d)))
        keep = max(1, min(context, int(context * rng.uniform(0.1, 1.0))))
        return dict(kind=kind, requests=n, context=context, keep=keep, sink=rng.choice([0, 1, 4]),
                    recent=rng.choice([0, 16, 128]), Hkv=Hkv, d=d, page=page)
    vocab = _log_int(rng, 1000, 200000)
    rows = _log_int(rng, 1, max(1, min(256, 256 * 131072 * 2 // (vocab * size))))
    return dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, filters=rng.choice(["none", "all", "mixed"]))


def _rows(c):
    """New rows of each request: the case's for the first, fewer for the later ones."""
    n, m = c["requests"], c["rows"]
    return [max(1, m - r * m // (2 * n)) for r in range(n)]


def _lens(c):
    """Tokens of each request, the step's rows included: from the case's number down to a quarter
    of it; in batches of four and more the last request is empty (a padding entry)."""
    n, top = c["requests"], c["context"]
    lens = [max(1, top - r * top * 3 // (4 * n)) for r in range(n)]
    if c["kind"] == "weigh":
        lens = [max(x, m) for x, m in zip(lens, _rows(c))]
    elif c["keep"] * 10 >= c["context"] * 9:    # a budget that decoding keeps to: all requests are near it
        lens = [max(1, top - r % 7) for r in range(n)]
    if n >= 4:
        lens[-1] = 0
    return lens


def _sections(c):
    return [c["d"] // 8, 3 * c["d"] // 16, 3 * c["d"] // 16]


def _seen(c):
    """(row, token) pairs of all requests."""
    seen = 0
    for x, k in zip(_lens(c), _rows(c)):
        k = min(k, x)
        seen += k * x - k * (k - 1) // 2 if c["causal"] else k * x
    return seen


def work(case):
    c = case
    size = 2 if c.get("dtype") == "bf16" else 4
    if c["kind"] in ("turn", "back"):
        n = c["rows"] * (c["Hq"] + c["Hkv"]) * c["d"]
        if c["kind"] == "turn":
            return {"bytes": 2 * n * size + 12 * c["rows"] + 2 * c["d"] * size, "flops": 7 * n}
        return {"bytes": 3 * n * size + 12 * c["rows"] + 2 * c["d"] * (size + 4), "flops": 15 * n}
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * size + 28), "flops": 4 * c["rows"] * c["vocab"]}
    lens, Hkv, d = _lens(c), c["Hkv"], c["d"]
    pages = sum(-(-x // c["page"]) for x in lens)
    if c["kind"] == "weigh":
        m = _rows(c)
        old = sum(max(0, x - k) for x, k in zip(lens, m))
        return {"bytes": sum(lens) * Hkv * (d + 4) + 4 * old * Hkv + pages * (4 + 4 * Hkv)
                + sum(m) * c["Hq"] * (d * size + 4), "flops": 2 * _seen(c) * c["Hq"] * d}
    moved = sum(min(x, c["keep"]) for x in lens if x > c["keep"])
    return {"bytes": Hkv * (4 * sum(lens) + 4 * sum(min(x, c["keep"]) for x in lens) + moved * (4 * d + 8))
            + pages * 4, "flops": sum(lens) * Hkv + 4 * moved * Hkv * d}


# ---------------------------------------------------------------------------------------
# inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, dtype=torch.float32, device=DEV)


def _scale_of(amax):
    """The least power of two 2^e, e >= -126, with amax <= 448 * 2^e; 0 for amax 0."""
    m, k = torch.frexp(amax)
    e = torch.where(m <= 0.875, k - 9, k - 8).clamp(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.zeros_like(amax))


def _encode(x, scale):
    """e4m3 codes (uint8) of x / scale, to nearest even."""
    s = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (x / s).to(torch.float8_e4m3fn).view(torch.uint8)


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


def _table(c, g, lens):
    """A block table over shuffled pages; page 0 is no one's."""
    need = [-(-x // c["page"]) for x in lens]
    n_pages = sum(need) + 3
    table = torch.zeros((len(lens), max(1, max(need))), dtype=torch.int32, device=DEV)
    order = (torch.randperm(n_pages - 1, generator=g, device=DEV) + 1).to(torch.int32)
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = order[at:at + k]
        at += k
    return table, n_pages


def _codes(g, n_pages, c, wide):
    """Codes and scales of a pool; pages differ in size, with `wide` some channels are ten times as wide."""
    x = _normal(g, n_pages, c["Hkv"], c["page"], c["d"])
    if wide:
        x[..., ::50] *= 10.0
    x *= torch.exp2(_normal(g, n_pages, c["Hkv"], 1, 1))
    x[..., 0, :] *= 0.01
    scale = _scale_of(x.abs().amax(dim=(2, 3)))
    return _encode(x, scale[:, :, None, None]), scale


def _pages_of(s, r, length):
    """Pages of request r and the shape to see them as tokens."""
    return s["table"][r, :-(-length // s["case"]["page"])].long()


def _keys(s, r, length):
    """Key rows [Hkv][length][d] of request r in 32 bits."""
    ids = _pages_of(s, r, length)
    k = _decode(s["K_codes"][ids], s["K_scale"][ids][..., None, None])
    return k.transpose(0, 1).flatten(1, 2)[:, :length]


def _query(s, at, m):
    """Rows at .. at + m - 1 as [Hkv][m * G][d] in 32 bits."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    return s["q"][at:at + m].float().view(m, c["Hkv"], G, c["d"]).transpose(0, 1).reshape(c["Hkv"], m * G, c["d"])


def _scores(s, r, length, m, at):
    """Scores [Hkv][m * G][length] of request r, -inf where a row does not see a token."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    x = torch.matmul(_query(s, at, m), _keys(s, r, length).transpose(1, 2)).mul_(1.0 / math.sqrt(c["d"]))
    if c["causal"]:
        last = (length - m + torch.arange(m, device=DEV)).repeat_interleave(G)
        x.masked_fill_(torch.arange(length, device=DEV) > last[:, None], float("-inf"))
    return x


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=dict(case))
    {"turn": _prepare_rows, "back": _prepare_rows, "weigh": _prepare_weigh, "evict": _prepare_evict,
     "sample": _prepare_sample}[c["kind"]](c, g, s)
    return s


def _prepare_rows(c, g, s):
    dt = TYPES[c["dtype"]]
    rows, Hq, Hkv, d = c["rows"], c["Hq"], c["Hkv"], c["d"]
    # the fused projection's output: a row holds its query, key and value heads
    qkv = _normal(g, rows, Hq + 2 * Hkv, d)
    qkv *= torch.exp2(_normal(g, 1, Hq + 2 * Hkv, 1))
    start = torch.randint(0, 1000, (1,), generator=g, device=DEV, dtype=torch.int32)
    s.update(qkv=qkv.to(dt), positions=_video_positions(rows) + start,
             q_weight=(1.0 + 0.3 * _normal(g, d)).to(dt), k_weight=(1.0 + 0.3 * _normal(g, d)).to(dt))
    if c["kind"] == "turn":
        s.update(q_out=torch.empty((rows, Hq, d), dtype=dt, device=DEV),
                 k_out=torch.empty((rows, Hkv, d), dtype=dt, device=DEV))
    else:
        s.update(q_out_grad=_normal(g, rows, Hq, d).to(dt), k_out_grad=_normal(g, rows, Hkv, d).to(dt),
                 qkv_grad=torch.empty((rows, Hq + 2 * Hkv, d), dtype=dt, device=DEV),
                 q_weight_grad=torch.empty(d, dtype=torch.float32, device=DEV),
                 k_weight_grad=torch.empty(d, dtype=torch.float32, device=DEV))
    if own:
        from paper_2608_24063_gb300 import viscache as vc
        s["rope"] = vc.make_rope(_sections(c), THETA, interleaved=c["order"] == "interleaved",
                                 adjacent=c["pairing"] == "adjacent")
        if c["kind"] == "back":
            s["ws"] = torch.empty(vc.viscache_norm_mrope_grad_workspace_size(rows, Hq, Hkv, d), dtype=torch.uint8,
                                  device=DEV)


def _prepare_weigh(c, g, s):
    lens, rows = _lens(c), _rows(c)
    table, n_pages = _table(c, g, lens)
    codes, scale = _codes(g, n_pages, c, True)
    # slots that no token was written to hold what was there before, NaN codes among it
    have = torch.zeros(n_pages, dtype=torch.int64, device=DEV)
    for r, x in enumerate(lens):
        k = -(-x // c["page"])
        if k:
            have[table[r, :k].long()] = c["page"]
            have[table[r, k - 1].long()] = x - (k - 1) * c["page"]
    live = (torch.arange(c["page"], device=DEV) < have[:, None])[:, None, :, None]
    codes = torch.where(live, codes, torch.full_like(codes, 0x7F))
    start = [0]
    for m in rows:
        start.append(start[-1] + m)
    total = start[-1]
    s.update(K_codes=codes, K_scale=scale, V_codes=torch.zeros_like(codes), V_scale=torch.zeros_like(scale),
             table=table, rows=total, seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
             row_start=torch.tensor(start, dtype=torch.int32, device=DEV),
             q=_normal(g, total, c["Hq"], c["d"]).to(TYPES[c["dtype"]]),
             # what earlier steps have added up
             weights=_uniform(g, n_pages, c["Hkv"], c["page"]).square_() * 4.0)
    # the attention's log-sum-exp of each row, which a program has from the call before
    lse = torch.full((total, c["Hq"]), float("-inf"), dtype=torch.float32, device=DEV)
    for r, (x, m) in enumerate(zip(lens, rows)):
        if x:
            z = torch.logsumexp(_scores(s, r, x, m, start[r]), dim=-1)                  # [Hkv][m * G]
            lse[start[r]:start[r + 1]] = z.view(c["Hkv"], m, -1).transpose(0, 1).reshape(m, c["Hq"])
    s["lse"] = lse
    if own:
        from paper_2608_24063_gb300 import viscache as vc
        s["cache"] = vc.Kv8Cache(codes, s["V_codes"], scale, s["V_scale"])
        s["step"] = vc.Kv8Step(table, s["seq_lens"], s["row_start"], total)
        s["ws"] = torch.empty(vc.viscache_kv8_workspace_size(total, c["Hq"], c["Hkv"], c["d"]), dtype=torch.uint8,
                              device=DEV)


def _prepare_evict(c, g, s):
    lens, n = _lens(c), c["requests"]
    table, n_pages = _table(c, g, lens)
    kc, ks = _codes(g, n_pages, c, True)
    vc_, vs = _codes(g, n_pages, c, False)
    s.update(K_codes=kc, K_scale=ks, V_codes=vc_, V_scale=vs, table=table,
             seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
             row_start=torch.arange(n + 1, dtype=torch.int32, device=DEV),
             keep=torch.full((n,), c["keep"], dtype=torch.int32, device=DEV),
             # a few tokens hold most of the weight
             weights=torch.exp2(3.0 * _normal(g, n_pages, c["Hkv"], c["page"])),
             kept=torch.zeros((n, c["Hkv"], c["keep"]), dtype=torch.int32, device=DEV),
             new_lens=torch.zeros(n, dtype=torch.int32, device=DEV))
    if own:
        from paper_2608_24063_gb300 import viscache as vc
        s["cache"] = vc.Kv8Cache(kc, vc_, ks, vs)
        s["step"] = vc.Kv8Step(table, s["seq_lens"], s["row_start"], n)
        s["ws"] = torch.empty(vc.viscache_kv8_evict_workspace_size(n, c["Hkv"]), dtype=torch.uint8, device=DEV)


def _prepare_sample(c, g, s):
    n, V = c["rows"], c["vocab"]
    wide = V + -V % 8                                   # the head's rows are padded to whole 16-byte pieces
    logits = (_normal(g, n, wide) * 2.5).to(TYPES[c["dtype"]])
    # a few tokens stand out in each row
    best = torch.randint(0, V, (n, 20), generator=g, device=DEV)
    logits.scatter_add_(1, best, (6.0 * _uniform(g, n, 20) + 4.0).to(logits.dtype))
    s.update(logits=logits[:, :V], u=_uniform(g, n), temperature=0.5 + _uniform(g, n),
             top_k=None, top_p=None, min_p=None, token=torch.empty(n, dtype=torch.int32, device=DEV),
             logprob=torch.empty(n, dtype=torch.float32, device=DEV))
    if c["filters"] != "none":
        s["top_k"] = torch.full((n,), 50, dtype=torch.int32, device=DEV)
        s["top_p"] = torch.full((n,), 0.95, dtype=torch.float32, device=DEV)
        s["min_p"] = torch.full((n,), 0.02, dtype=torch.float32, device=DEV)
    if c["filters"] == "mixed":
        # requests with settings of their own: some greedy, some with one filter, some with none
        turn = torch.arange(n, device=DEV) % 5
        s["temperature"][turn == 0] = 0.0
        s["top_k"][turn >= 2] = 0
        s["top_p"] = torch.where(turn == 3, torch.ones_like(s["top_p"]), 0.5 + 0.49 * _uniform(g, n))
        s["min_p"][turn >= 2] = 0.0


# ---------------------------------------------------------------------------------------
# one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"turn": _plain_turn, "back": _plain_back, "weigh": _plain_weigh, "evict": _plain_evict,
            "sample": _plain_sample}[kind](state)


def _own(kind, s):
    from paper_2608_24063_gb300 import viscache as vc
    c = s["case"]
    if kind in ("turn", "back"):
        Hq, Hkv = c["Hq"], c["Hkv"]
        q, k = s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + Hkv]
        if kind == "turn":
            vc.viscache_norm_mrope(s["rope"], s["positions"], q, k, s["q_weight"], s["k_weight"], eps=EPS,
                                   q_out=s["q_out"], k_out=s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        dq, dk = s["qkv_grad"][:, :Hq], s["qkv_grad"][:, Hq:Hq + Hkv]
        vc.viscache_norm_mrope_grad(s["rope"], s["positions"], q, k, s["q_out_grad"], s["k_out_grad"], s["q_weight"],
                                    s["k_weight"], eps=EPS, q_grad=dq, k_grad=dk, q_weight_grad=s["q_weight_grad"],
                                    k_weight_grad=s["k_weight_grad"], ws=s["ws"])
        return {"q": dq, "k": dk, "q_weight": s["q_weight_grad"], "k_weight": s["k_weight_grad"]}
    if kind == "weigh":
        vc.viscache_kv8_weigh(s["cache"], s["step"], s["q"], s["lse"], s["weights"], causal=c["causal"], ws=s["ws"])
        return {"weights": s["weights"]}
    if kind == "evict":
        vc.viscache_kv8_evict(s["cache"], s["step"], s["weights"], s["keep"], c["keep"], sink=c["sink"],
                              recent=c["recent"], kept=s["kept"], new_lens=s["new_lens"], ws=s["ws"])
        return _evicted(s)
    vc.viscache_sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], token=s["token"],
                       logprob=s["logprob"])
    return {"token": s["token"], "logprob": s["logprob"]}


def _evicted(s):
    """The cache's codes as the 8-bit numbers they are, scales, weights, and what was kept."""
    return {"K": s["K_codes"].view(torch.float8_e4m3fn), "K_scale": s["K_scale"],
            "V": s["V_codes"].view(torch.float8_e4m3fn), "V_scale": s["V_scale"], "weights": s["weights"],
            "kept": s["kept"], "lens": s["new_lens"]}


def _axis_of(c):
    """The axis whose position turns frequency i of d / 2."""
    sec, half = _sections(c), c["d"] // 2
    i = torch.arange(half, device=DEV)
    if c["order"] == "interleaved":     # i mod 3 while that axis has frequencies left, axis 0 after
        a = i % 3
        return torch.where(i < 3 * torch.tensor(sec, device=DEV)[a], a, torch.zeros_like(a))
    return (i >= sec[0]).long() + (i >= sec[0] + sec[1]).long()


def _angles(s):
    """Cosines and sines [rows][1][half]; the phase in turns as a 40-bit fraction."""
    c = s["case"]
    half = c["d"] // 2
    i = torch.arange(half, dtype=torch.float64, device=DEV)
    f = (THETA ** (-i / half) / (2 * math.pi) * 2.0 ** 40).round().to(torch.int64)
    p = s["positions"].to(torch.int64)[_axis_of(c)].t()
    angle = ((p * f) & ((1 << 40) - 1)).to(torch.float32) * (2 * math.pi / 2.0 ** 40)
    return angle.cos()[:, None, :], angle.sin()[:, None, :]


def _rotate(x, cos, sin, pairing):
    if pairing == "halves":
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)


def _plain_turn(s):
    c = s["case"]
    cos, sin = _angles(s)
    out = {}
    for name, x in (("q", s["qkv"][:, :c["Hq"]]), ("k", s["qkv"][:, c["Hq"]:c["Hq"] + c["Hkv"]])):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * s[name + "_weight"].float()
        out[name] = _rotate(x, cos, sin, c["pairing"]).to(s["qkv"].dtype)
    return out


def _plain_back(s):
    c = s["case"]
    cos, sin = _angles(s)
    out = {}
    for name, x in (("q", s["qkv"][:, :c["Hq"]]), ("k", s["qkv"][:, c["Hq"]:c["Hq"] + c["Hkv"]])):
        x = x.float()
        r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
        g = _rotate(s[name + "_out_grad"].float(), cos, -sin, c["pairing"])
        n = x * r
        out[name + "_weight"] = (g * n).sum(dim=(0, 1))
        g = g * s[name + "_weight"].float()
        out[name] = (r * (g - n * (g * n).mean(dim=-1, keepdim=True))).to(s["qkv"].dtype)
    return out


def _plain_weigh(s):
    c = s["case"]
    page = c["page"]
    at = 0
    for r, (length, m) in enumerate(zip(_lens(c), _rows(c))):
        if length:
            x = _scores(s, r, length, m, at)
            lse = s["lse"][at:at + m].view(m, c["Hkv"], -1).transpose(0, 1).reshape(c["Hkv"], -1)
            a = x.sub_(lse[..., None]).exp_().sum(dim=1)                                # [Hkv][length]
            del x
            ids = _pages_of(s, r, length)
            there = s["weights"][ids].transpose(0, 1).flatten(1)                        # [Hkv][pages * page]
            new = there.clone()
            old = length - m
            new[:, :old] += a[:, :old]
            new[:, old:length] = a[:, old:]
            s["weights"][ids] = new.view(c["Hkv"], len(ids), page).transpose(0, 1)
        at += m
    return {"weights": s["weights"]}


def _order(w, length, c):
    """Tokens [Hkv][length] by weight, the largest first; protected ones before all others."""
    w = w[:, :length].clone()
    w[:, :c["sink"]] = float("inf")
    w[:, max(0, length - c["recent"]):] = float("inf")
    return torch.sort(w, dim=1, descending=True, stable=True)[1]


def _plain_evict(s):
    c = s["case"]
    page, Hkv, k = c["page"], c["Hkv"], c["keep"]
    heads = torch.arange(Hkv, device=DEV)[:, None]
    for r, length in enumerate(_lens(c)):
        new = min(length, k)
        s["new_lens"][r] = new
        if new == length:
            s["kept"][r, :, :new] = torch.arange(new, dtype=torch.int32, device=DEV)
            continue
        ids = _pages_of(s, r, length)
        w = s["weights"][ids].transpose(0, 1).flatten(1)
        kept = torch.sort(_order(w, length, c)[:, :k], dim=1)[0]                        # [Hkv][k]
        s["kept"][r, :, :k] = kept.to(torch.int32)
        gap = (kept == torch.arange(k, device=DEV)).sum(dim=1)                          # the first evicted token
        n = -(-k // page)
        slots = torch.arange(n * page, device=DEV)
        written = (slots >= gap[:, None] // page * page) & (slots < k)                  # [Hkv][slots]
        src = torch.nn.functional.pad(kept, (0, n * page - k))
        sp, ss = ids[src // page], src % page                                           # source page and slot
        to = ids[:n]
        written_pages = written.view(Hkv, n, page).any(dim=2).t()                       # [n][Hkv]
        written = written.view(Hkv, n, page).transpose(0, 1)                            # [n][Hkv][page]
        moved = s["weights"][sp, heads, ss].view(Hkv, n, page).transpose(0, 1)
        weights = torch.where(written, moved, s["weights"][to])
        for codes, scale in ((s["K_codes"], s["K_scale"]), (s["V_codes"], s["V_scale"])):
            x = _decode(codes[sp, heads, ss], scale[sp, heads][..., None])
            x = x.view(Hkv, n, page, c["d"]).transpose(0, 1)                            # [n][Hkv][page][d]
            amax = torch.where(written[..., None], x.abs(), torch.zeros_like(x)).amax(dim=(2, 3))
            now = _scale_of(amax)
            out = torch.where(written[..., None], _encode(x, now[..., None, None]), codes[to])
            codes[to] = out
            scale[to] = torch.where(written_pages, now, scale[to])
        s["weights"][to] = weights
    return _evicted(s)


def _plain_sample(s):
    # in 64 bits: a random number may lie next to a border between two tokens
    x = s["logits"].double()
    n, V = x.shape
    T = s["temperature"].double()[:, None]
    y, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((y - y[:, :1]) / torch.where(T > 0, T, torch.ones_like(T)))
    rank = torch.arange(V, device=DEV)
    live = (T > 0) | (rank == 0)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        live = live & ((k <= 0) | (rank < k))
    w = torch.where(live, w, torch.zeros_like(w))
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = w.cumsum(dim=1) - w
        live = live & ((p >= 1) | (before < p * w.sum(dim=1, keepdim=True)) | (rank == 0))
    if s["min_p"] is not None:
        live = live & (w >= s["min_p"].double()[:, None].clamp(max=1.0))
    w = torch.where(live, w, torch.zeros_like(w))
    mass = torch.zeros_like(w).scatter_(1, order, w)                                    # in order of the tokens
    cum = mass.cumsum(dim=1)
    total = cum[:, -1:]
    token = torch.searchsorted(cum, s["u"].double()[:, None] * total, right=True)
    # past the last token with any mass there is nothing to draw
    last = torch.where(mass > 0, rank, torch.zeros_like(rank)).amax(dim=1, keepdim=True)
    token = torch.minimum(token, last)
    logprob = torch.log(mass.gather(1, token) / total)
    return {"token": token[:, 0].to(torch.int32), "logprob": logprob[:, 0].float()}


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
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"turn": _exact_rows, "back": _exact_rows, "weigh": _exact_weigh, "evict": _exact_evict,
            "sample": _exact_sample}[case["kind"]](case, s)


def _exact_rows(c, s):
    f64 = torch.float64
    half, sec = c["d"] // 2, _sections(c)
    out = {}
    for name, lo, hi in (("q", 0, c["Hq"]), ("k", c["Hq"], c["Hq"] + c["Hkv"])):
        x, weight = s["qkv"][:, lo:hi].to(f64), s[name + "_weight"].to(f64)
        r = 1.0 / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / c["d"] + EPS)
        back = c["kind"] == "back"
        z = s[name + "_out_grad"].to(f64) if back else x * r * weight
        y = torch.empty_like(z)
        for i in range(half):
            if c["order"] == "interleaved":
                a = i % 3 if i < 3 * sec[i % 3] else 0
            else:
                a = 0 if i < sec[0] else 1 if i < sec[0] + sec[1] else 2
            w = s["positions"][a].to(f64) * (THETA ** (-i / half)) * (-1.0 if back else 1.0)
            co, si = torch.cos(w)[:, None], torch.sin(w)[:, None]
            u, v = (i, i + half) if c["pairing"] == "halves" else (2 * i, 2 * i + 1)
            y[..., u] = z[..., u] * co - z[..., v] * si
            y[..., v] = z[..., u] * si + z[..., v] * co
        if not back:
            out[name] = y
            continue
        out[name + "_weight"] = (y * x * r).sum(dim=(0, 1))
        h = y * weight
        out[name] = h * r - x * r ** 3 * ((h * x).sum(dim=-1, keepdim=True) / c["d"])
    return out


def _exact_weigh(c, s):
    value, f64 = _e4m3_table(), torch.float64
    Hq, Hkv, d, G, page = c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"], c["page"]
    out = s["weights"].to(f64)
    at = 0
    for r, (length, m) in enumerate(zip(_lens(c), _rows(c))):
        ids = s["table"][r, :-(-length // page)].long()
        t = torch.arange(length, device=DEV)
        for g in range(Hkv if length else 0):
            k = (value[s["K_codes"][ids, g].long()] * s["K_scale"][ids, g].to(f64)[:, None, None])
            k = k.reshape(-1, d)[:length]
            total = torch.zeros(length, dtype=f64, device=DEV)
            for h in range(g * G, (g + 1) * G):
                x = s["q"][at:at + m, h].to(f64) @ k.T / math.sqrt(d)
                p = torch.exp(x - s["lse"][at:at + m, h].to(f64)[:, None])
                if c["causal"]:
                    p = torch.where(t <= length - m + torch.arange(m, device=DEV)[:, None], p, 0.0)
                total += p.sum(dim=0)
            was = out[ids[t // page], g, t % page]
            out[ids[t // page], g, t % page] = torch.where(t < length - m, was, 0.0) + total
        at += m
    return {"weights": out}


def _exact_evict(c, s):
    if c["requests"] * c["Hkv"] * -(-c["keep"] // c["page"]) > 20000:
        return None
    value, f64, page = _e4m3_table(), torch.float64, c["page"]
    pools = [(value[s[n + "_codes"].long()], s[n + "_scale"].to(f64)) for n in ("K", "V")]
    weights, kept_out = s["weights"].to(f64), torch.zeros_like(s["kept"])
    lens = []
    for r, length in enumerate(_lens(c)):
        new = min(length, c["keep"])
        lens.append(new)
        ids = s["table"][r, :-(-length // page)].long()
        for g in range(c["Hkv"] if length else 0):
            w = s["weights"][ids, g].flatten()[:length].tolist()
            first = lambda t: t < c["sink"] or t >= length - c["recent"]
            order = sorted(range(length), key=lambda t: (-math.inf if first(t) else -w[t], t))
            kept = sorted(order[:new])
            kept_out[r, g, :new] = torch.tensor(kept, dtype=torch.int32, device=DEV)
            gap = next((i for i, t in enumerate(kept) if i != t), new)
            if new == length:
                continue
            t = torch.tensor(kept, device=DEV)
            sp, ss = ids[t // page], t % page
            moved = weights[sp, g, ss]
            held = [(v[sp, g, ss], sc[sp, g]) for v, sc in pools]
            for j in range(gap // page, -(-new // page)):
                a, b, p = j * page, min(new, (j + 1) * page), ids[j]
                weights[p, g, :b - a] = moved[a:b]
                for (v, sc), (hv, hs) in zip(pools, held):
                    y = hv[a:b] * hs[a:b, None]
                    amax = float(y.abs().max())
                    now = 2.0 ** max(-126, math.ceil(math.log2(amax / 448.0))) if amax > 0 else 0.0
                    v[p, g, :b - a] = _round_e4m3(y / (now if now > 0 else 1.0))
                    sc[p, g] = now
    return {"K": pools[0][0], "K_scale": pools[0][1], "V": pools[1][0], "V_scale": pools[1][1], "weights": weights,
            "kept": kept_out, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}


def _exact_sample(c, s):
    token, logprob = [], []
    rows = s["logits"].double()
    for r in range(c["rows"]):
        x = rows[r]
        T, u = float(s["temperature"][r]), float(s["u"][r])
        if T <= 0.0:
            token.append(int(torch.nonzero(x == x.max())[0]))
            logprob.append(0.0)
            continue
        w = torch.exp((x - x.max()) / T)
        order = torch.argsort(-x, stable=True)
        n = c["vocab"]
        if s["top_k"] is not None and int(s["top_k"][r]) > 0:
            n = min(n, int(s["top_k"][r]))
        if s["top_p"] is not None and float(s["top_p"][r]) < 1.0:
            cum = w[order[:n]].cumsum(0)
            n = min(n, int((cum < float(s["top_p"][r]) * cum[-1]).sum()) + 1)
        if s["min_p"] is not None:
            n = min(n, max(1, int((w >= float(s["min_p"][r])).sum())))
        kept = torch.sort(order[:n])[0]
        cum = w[kept].cumsum(0)
        i = min(int((cum <= u * cum[-1]).sum()), n - 1)
        token.append(int(kept[i]))
        logprob.append(float(torch.log(w[kept[i]] / cum[-1])))
    return {"token": torch.tensor(token, dtype=torch.int32, device=DEV),
            "logprob": torch.tensor(logprob, dtype=torch.float64, device=DEV)}
