"""The serving operators between the projections and the next token, as timed cases.

Four operators of the library that a decoding program calls one after another
around its W8A8 products: the rotation of query and key heads by their position,
the append of a fused QKV projection's rows to a paged key/value cache (rotation,
INT8 or bf16 rows), the attention of new tokens over that cache (single tokens and
chunks), and the draw of the next token from the lm_head's logits.

Where ``own`` is false, ``run`` computes the same with elementary torch operations
in binary32 (angles, and the weights that decide a draw, in binary64); ``exact``
follows the definitions in binary64, written apart.

Shapes are those of Gemma-3-1B (4 query heads on 1 key/value head of 256,
vocabulary 262144) and generic ones.  Keys, values and queries are N(0, 1.5^2)
with a few strong channels; logits are N(0, 2.5^2) with a handful of likely tokens.
"""

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"

# (query heads, key/value heads, head width)
HEADS = [(4, 1, 256), (4, 1, 256), (8, 4, 256), (16, 8, 128), (16, 2, 128), (2, 2, 256), (6, 2, 128)]
# (heads, head width) rotated by themselves
ROTATED = [(5, 256), (5, 256), (18, 128), (6, 128), (10, 256)]
VOCABS = [262144, 262144, 32001, 100003, 65536]


def listed():
    return [
        # one token's query heads and key head, in its fused QKV row, before the one-token attention
        {"name": "rope_1", "kind": "rope", "rows": 1, "heads": 5, "d": 256, "rot": 256, "layout": "half", "scaling": "linear", "dt": "bf16"},
        # a ragged prompt's heads in binary32, half of each head rotated in neighbouring pairs, scaled for long contexts
        {"name": "rope_part_4095", "kind": "rope", "rows": 4095, "heads": 18, "d": 128, "rot": 64, "layout": "interleaved", "scaling": "yarn", "dt": "f32"},
        # one decode step of a batch: rotate, quantise and store each sequence's new row
        {"name": "append_int8_48", "kind": "append", "seqs": 48, "new": 1, "mix": "same", "ctx": 4096, "heads": 4, "kv": 1, "d": 256, "int8": True, "page": 64, "window": 0, "pad": 0},
        # prompts of three requests stored in a bf16 cache
        {"name": "append_bf16_2039", "kind": "append", "seqs": 3, "new": 2039, "mix": "ragged", "ctx": 4096, "heads": 8, "kv": 4, "d": 256, "int8": False, "page": 16, "window": 0, "pad": 0},
        # one request's decode step
        {"name": "decode_1", "kind": "attn", "seqs": 1, "new": 1, "mix": "same", "ctx": 2500, "heads": 4, "kv": 1, "d": 256, "int8": True, "page": 64, "window": 0, "pad": 0},
        # a decode batch of requests of very different lengths
        {"name": "decode_64", "kind": "attn", "seqs": 64, "new": 1, "mix": "same", "ctx": 16384, "heads": 4, "kv": 1, "d": 256, "int8": True, "page": 64, "window": 0, "pad": 0},
        # a sliding-window layer of a batch that checks a few drafted tokens; pages behind the window are given back
        {"name": "window_bf16_40", "kind": "attn", "seqs": 40, "new": 4, "mix": "ragged", "ctx": 9000, "heads": 8, "kv": 4, "d": 256, "int8": False, "page": 32, "window": 1024, "pad": 3},
        # a chunk of one request's prompt beside the decode steps of others
        {"name": "mixed_int8_12", "kind": "attn", "seqs": 12, "new": 509, "mix": "one", "ctx": 8192, "heads": 16, "kv": 8, "d": 128, "int8": True, "page": 16, "window": 0, "pad": 5},
        # a long prompt attended at once
        {"name": "prompt_bf16_8192", "kind": "attn", "seqs": 1, "new": 8192, "mix": "same", "ctx": 8192, "heads": 4, "kv": 1, "d": 256, "int8": False, "page": 64, "window": 0, "pad": 0},
        # the next token of one request, every filter on
        {"name": "sample_1", "kind": "sample", "rows": 1, "n": 262144, "dt": "bf16", "mode": "all"},
        # the next tokens of a decode batch, nucleus only
        {"name": "sample_64", "kind": "sample", "rows": 64, "n": 262144, "dt": "bf16", "mode": "top_p"},
        # binary32 logits of an odd vocabulary, temperature and a floor on the probability
        {"name": "sample_f32_131", "kind": "sample", "rows": 131, "n": 100003, "dt": "f32", "mode": "min_p"},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    kind = rng.choice(["rope", "append", "attn", "attn", "attn", "sample", "sample"])
    if kind == "rope":
        heads, d = rng.choice(ROTATED)
        return {"kind": kind, "rows": _spread(rng, 1, 16384), "heads": heads, "d": d, "rot": rng.choice([d, d, d // 2, d // 4]),
                "layout": rng.choice(["half", "half", "interleaved"]), "scaling": rng.choice(["none", "linear", "ntk", "yarn"]),
                "dt": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "sample":
        return {"kind": kind, "rows": _spread(rng, 1, 256), "n": rng.choice(VOCABS), "dt": rng.choice(["bf16", "bf16", "bf16", "f32"]),
                "mode": rng.choice(["all", "all", "top_k", "top_p", "min_p", "none"])}
    heads, kv, d = rng.choice(HEADS)
    seqs = _spread(rng, 1, 64)
    new = rng.choice([1, 1, rng.randint(2, 8), _spread(rng, 9, 4096)])
    ctx = max(new, _spread(rng, 64, 32768))
    return {"kind": kind, "seqs": seqs, "new": new, "mix": rng.choice(["same", "ragged", "one"]) if new > 1 else "same", "ctx": ctx,
            "heads": heads, "kv": kv, "d": d, "int8": rng.random() < 0.6, "page": rng.choice([16, 32, 64, 128]),
            "window": rng.choice([0, 0, 512, 1024]) if kind == "attn" else 0, "pad": rng.choice([0, 0, 3]) if kind == "attn" else 0}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _plain_scores(case):
    """Scores that the padded plain form holds at once."""
    return case["seqs"] * case["heads"] * case["new"] * case["ctx"] if case["kind"] == "attn" else 0


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _drawn(rng)
        if _cost(case) <= most and _plain_scores(case) <= 1 << 29:
            return case


# ------------------------------------------------------------------ lengths and inputs

def _lengths(case):
    """New tokens and contexts (with them) of a case's sequences: its own, whatever the seed."""
    r = random.Random("%(seqs)d %(new)d %(mix)s %(ctx)d %(heads)d %(page)d" % case)
    n, new, ctx = case["seqs"], case["new"], case["ctx"]
    fresh = {"same": [new] * n, "one": [new] + [1] * (n - 1), "ragged": [new] + [r.randint(0, new) for _ in range(n - 1)]}[case["mix"]]
    total = [ctx] + [max(f, _spread(r, max(1, ctx // 8), ctx)) for f in fresh[1:]]
    return fresh, total


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _normal(g, shape, sigma, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def _frequencies(rot, scaling):
    """Radians a position for each pair, and the factor on cosine and sine."""
    base, factor, original = 1e6 if scaling in ("none", "linear") else 1e4, 8.0, 4096.0
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "ntk" and rot > 2:
        base *= factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":  # pairs that turn often in the original context keep their speed, slow ones are slowed by the factor
        lo, hi = (rot * math.log(original / (turns * 2.0 * math.pi)) / (2.0 * math.log(base)) for turns in (32.0, 1.0))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
        slow = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f * (1.0 - slow) + f / factor * slow, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _heads(g, shape, sigma=1.5):
    """bf16 heads, the last axis a head, with a few strong channels."""
    x = torch.randn(shape, generator=g, device=DEV) * sigma
    x[..., torch.randperm(shape[-1], generator=g, device=DEV)[:4]] *= 3.0
    return x.to(torch.bfloat16)


def _codes(x):
    """INT8 codes and binary32 scales of rows: s = max |x| / 127, codes rne(x / s)."""
    s = x.abs().amax(-1) / 127.0
    return torch.where(s[..., None] > 0, x / s[..., None], torch.zeros_like(x)).round().clamp(-127, 127), s


def _paged(case, g):
    fresh, total = _lengths(case)
    page, window = case["page"], case["window"]
    # a page that ends before the first new token's window has been given back
    first = [max(0, t - f + 1 - window) // page if window else 0 for f, t in zip(fresh, total)]
    blocks = [-(-t // page) for t in total]
    n_pages = sum(b - f for b, f in zip(blocks, first)) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = np.full((len(fresh), max(blocks)), -1, np.int64)
    at = 0
    for s, (b, f) in enumerate(zip(blocks, first)):
        table[s, f:b] = np.arange(at, at + b - f)
        at += b - f
    where = torch.from_numpy(table).to(DEV)
    table = torch.where(where >= 0, order[where.clamp_min(0)], -1).int()
    shape = (n_pages, case["kv"], page, case["d"])
    s = {"table": table, "ctx_len": torch.tensor(total, dtype=torch.int32, device=DEV),
         "q_start": torch.tensor(np.cumsum([0] + fresh), dtype=torch.int32, device=DEV),
         "max_q": max(fresh), "rows": sum(fresh) + case["pad"]}
    for name in "kv":
        x = _heads(g, shape)
        if case["int8"]:
            c, s["s" + name] = _codes(x.float())
            s[name] = c.to(torch.int8)
        else:
            s[name], s["s" + name] = x, None
    return s


def _dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "rope":
        freq, scale = _frequencies(case["rot"], case["scaling"])
        rows, heads, d = case["rows"], case["heads"], case["d"]
        x = _heads(g, (rows, heads + 1, d)).to(_dtype(case["dt"]))[:, :heads]  # the row goes on with the value head
        if case["dt"] == "f32":
            x = x * 1.01
        start = torch.randint(0, 100000, (1,), generator=g, device=DEV)
        pos = (start + torch.arange(rows, device=DEV)).int()
        return {"kind": kind, "case": case, "x": x, "pos": pos, "freq": torch.from_numpy(freq).to(DEV), "scale": scale}
    if kind == "sample":
        m, n, mode = case["rows"], case["n"], case["mode"]
        l = torch.randn((m, n), generator=g, device=DEV) * 2.5
        likely = torch.randint(0, n, (m, 24), generator=g, device=DEV)
        l.scatter_(1, likely, 9.0 + 2.5 * torch.randn((m, 24), generator=g, device=DEV))
        r = torch.rand((4, m), generator=g, device=DEV)
        s = {"kind": kind, "case": case, "logits": l.to(_dtype(case["dt"])), "u": r[0].contiguous(),
             "temperature": 0.6 + 0.8 * r[1], "top_k": None, "top_p": None, "min_p": None}
        if mode in ("all", "top_k"):
            s["top_k"] = (20 + 80 * r[2]).int()
        if mode in ("all", "top_p"):
            s["top_p"] = 0.8 + 0.19 * r[3]
        if mode in ("all", "min_p"):
            s["min_p"] = 0.002 + 0.05 * r[2]
        return s
    s = _paged(case, g)
    heads, kv, d = case["heads"], case["kv"], case["d"]
    s.update(kind=kind, case=case)
    if kind == "append":
        freq, scale = _frequencies(d, "linear")
        s.update(qkv=_heads(g, (s["rows"], heads + 2 * kv, d)).reshape(s["rows"], -1), freq=torch.from_numpy(freq).to(DEV), scale=scale)
    else:
        s.update(q=_heads(g, (s["rows"], heads, d), 0.7), out=torch.zeros((s["rows"], heads, d), dtype=torch.bfloat16, device=DEV))
    return s


# ------------------------------------------------------------------ the library's calls

def _run_own(s):
    from paper_2608_28003_amd import w8a8

    kind, case = s["kind"], s["case"]
    if kind == "rope":
        rope = w8a8.Rope(case["d"], case["rot"], case["layout"], s["freq"], s["scale"])
        return w8a8.rope(rope, s["x"], s["pos"])
    if kind == "sample":
        return w8a8.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    cache = w8a8.PagedKV(s["k"], s["v"], s["sk"], s["sv"])
    batch = w8a8.PagedBatch(s["table"], s["q_start"], s["ctx_len"], s["max_q"])
    if kind == "append":
        rope = w8a8.Rope(case["d"], case["d"], "half", s["freq"], s["scale"])
        q = w8a8.kv_append(s["qkv"], cache, batch, case["heads"], rope=rope)
        return [q, *w8a8.kv_read(cache, batch, s["rows"])]
    return w8a8.attn_paged(s["q"], cache, batch, window=case["window"] or None, out=s["out"])


# ------------------------------------------------------------------ the plain forms

def _rotate(x, pos, freq, scale, rot, layout):
    """x: [rows, heads, d] binary32."""
    angle = pos.double()[:, None] * freq
    c, s = (f(angle).float()[:, None] * scale for f in (torch.cos, torch.sin))
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., ::2], head[..., 1::2]) if layout == "interleaved" else (head[..., :rot // 2], head[..., rot // 2:])
    a, b = a * c - b * s, b * c + a * s
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if layout == "interleaved" else torch.cat([a, b], -1), rest], -1)


def _rows_of(s):
    """Sequence and position of every new token."""
    start, ctx = s["q_start"].long(), s["ctx_len"].long()
    row = torch.arange(s["rows"] - s["case"]["pad"], device=DEV)
    seq = torch.searchsorted(start, row, right=True) - 1
    return row, seq, ctx[seq] - (start[seq + 1] - row)


def _plain_append(s):
    case = s["case"]
    h, kv, d = case["heads"], case["kv"], case["d"]
    _, seq, pos = _rows_of(s)
    x = s["qkv"].float().view(-1, h + 2 * kv, d)
    qk = _rotate(x[:, :h + kv], pos, s["freq"], s["scale"], d, "half")
    page, slot = s["table"].long()[seq, pos // case["page"]], pos % case["page"]
    q, new = qk[:, :h].to(torch.bfloat16), [qk[:, h:], x[:, h + kv:]]
    if not case["int8"]:
        new = [v.to(torch.bfloat16) for v in new]
        s["k"][page, :, slot], s["v"][page, :, slot] = new
        return [q, *new]
    (ck, sk), (cv, sv) = (_codes(v) for v in new)
    s["k"][page, :, slot], s["v"][page, :, slot] = ck.to(torch.int8), cv.to(torch.int8)
    s["sk"][page, :, slot], s["sv"][page, :, slot] = sk, sv
    return [q, (ck * sk[..., None]).to(torch.bfloat16), (cv * sv[..., None]).to(torch.bfloat16)]


def _plain_attn(s):
    case = s["case"]
    n, h, kv, d, page = case["seqs"], case["heads"], case["kv"], case["d"], case["page"]
    start, ctx, table = s["q_start"].long(), s["ctx_len"].long(), s["table"].long()
    held, at, long = table >= 0, table.clamp_min(0), table.shape[1] * page

    def rows(x, scale):  # [seqs * kv, long, d]
        x = x[at].float() if scale is None else x[at].float() * scale[at][..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(n * kv, long, d)

    step = torch.arange(s["max_q"], device=DEV)
    fresh = (start[1:] - start[:-1])[:, None]
    row, used = start[:-1, None] + step, step < fresh
    q = s["q"][row.clamp_max(s["rows"] - 1)].float().view(n, -1, kv, h // kv, d).permute(0, 2, 3, 1, 4).reshape(n * kv, -1, d)
    score = torch.bmm(q, rows(s["k"], s["sk"]).transpose(1, 2)).mul_(d ** -0.5).view(n, h, -1, long)
    pos, key = (ctx[:, None] - fresh + step)[..., None], torch.arange(long, device=DEV)
    seen = (key <= pos) & held.repeat_interleave(page, 1)[:, None]
    if case["window"]:
        seen = seen & (key > pos - case["window"])
    score.masked_fill_(~seen[:, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.bmm(score.view(n * kv, -1, long), rows(s["v"], s["sv"])).view(n, h, -1, d)
    o = torch.where(total > 0, o / total, 0.0).transpose(1, 2)
    s["out"][row[used]] = o[used].to(torch.bfloat16)
    return s["out"]


def _plain_sample(s):
    l = s["logits"].double()
    l = torch.where(torch.isnan(l), -math.inf, l)
    m, n = l.shape
    t, u = s["temperature"].double()[:, None], s["u"].double()[:, None]
    top = l.amax(1, keepdim=True)
    w = torch.where(l == top, 1.0, torch.exp((l - top) / t)) * (l > -math.inf)
    order = torch.sort(l, dim=1, descending=True, stable=True).indices
    ranked, rank = w.gather(1, order), torch.arange(n, device=DEV)
    keep = (rank == 0) | (t > 0).expand(m, n)
    if s["top_k"] is not None:
        keep = keep & ((rank < s["top_k"][:, None]) | (s["top_k"][:, None] <= 0))
    if s["top_p"] is not None:
        cum = torch.cumsum(ranked * keep, 1)
        before = torch.cat([torch.zeros_like(cum[:, :1]), cum[:, :-1]], 1)
        p = s["top_p"].double()[:, None]
        keep = keep & ((before < p * cum[:, -1:]) | (p >= 1) | (rank == 0))
    if s["min_p"] is not None:
        keep = keep & ((ranked >= s["min_p"].double()[:, None]) | (rank == 0))
    kept = torch.zeros_like(w).scatter_(1, order, ranked * keep)
    cum = torch.cumsum(kept, 1)
    token = (cum <= u * cum[:, -1:]).sum(1).clamp_max(n - 1)
    return [token, (kept.gather(1, token[:, None]) / cum[:, -1:]).float().view(-1)]


def run(s):
    if own:
        return _run_own(s)
    kind = s["kind"]
    if kind == "rope":
        case = s["case"]
        return _rotate(s["x"].float(), s["pos"], s["freq"], s["scale"], case["rot"], case["layout"]).to(s["x"].dtype)
    return {"append": _plain_append, "attn": _plain_attn, "sample": _plain_sample}[kind](s)


# ------------------------------------------------------------------ what the path cannot do without

def work(case):
    kind = case["kind"]
    if kind == "rope":
        n = case["rows"] * case["heads"] * case["d"]
        return {"bytes": 2 * n * (2 if case["dt"] == "bf16" else 4) + 4 * case["rows"] + 4 * case["rot"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    if kind == "sample":
        n = case["rows"] * case["n"]
        return {"bytes": n * (2 if case["dt"] == "bf16" else 4) + 32 * case["rows"], "flops": 4 * n}
    fresh, total = _lengths(case)
    h, kv, d, w = case["heads"], case["kv"], case["d"], case["window"]
    row = 2 * kv * (d + 4 if case["int8"] else 2 * d)  # a token's key and value rows in the cache
    if kind == "append":  # the projection's rows in, queries and cached rows out, the cached rows read back as bf16
        rows = sum(fresh)
        return {"bytes": rows * (2 * (h + 2 * kv) * d + 2 * h * d + 2 * row + 4 * kv * d), "flops": 3 * rows * (h + kv) * d}
    pairs, keys = 0, 0
    for f, t in zip(fresh, total):
        if f:
            span = min(w, t) if w else t
            full = max(0, min(f, t - span + 1))  # tokens that see a whole window
            pairs += full * span + sum(range(t - f + 1, t - full + 1)) if w else f * t - f * (f - 1) // 2
            keys += min(t, span + f - 1) if w else t
    return {"bytes": keys * row + 4 * sum(fresh) * h * d, "flops": 4 * pairs * h * d}


# ------------------------------------------------------------------ the same in 64 bits

def _turned(x, pos, freq, scale, rot, layout):
    """Each pair of a head as a complex number times e^(i angle)."""
    x = x.double()
    turn = torch.polar(torch.full_like(pos, scale, dtype=torch.float64)[:, None].expand(-1, rot // 2).contiguous(), pos.double()[:, None] * freq)[:, None]
    out = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if layout == "interleaved" else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_sample(s):
    """Probability that each row's token is drawn with; the token is given by the definition alone."""
    logits, got = s["logits"].double().cpu().numpy(), []
    col = {k: None if s[k] is None else s[k].double().cpu().numpy() for k in ("temperature", "u", "top_k", "top_p", "min_p")}
    for i, l in enumerate(logits):
        by = np.argsort(-l, kind="stable")
        w = np.exp((l[by] - l[by[0]]) / col["temperature"][i])
        if col["top_k"] is not None:
            w = w[:int(col["top_k"][i])]
        if col["top_p"] is not None:
            c = np.cumsum(w)
            w = w[:int(np.searchsorted(c, col["top_p"][i] * c[-1], side="left")) + 1]
        if col["min_p"] is not None:
            w = w[:max(1, int((w >= col["min_p"][i]).sum()))]
        by = by[:len(w)]
        back = np.argsort(by)
        c = np.cumsum(w[back])
        at = min(int(np.searchsorted(c, col["u"][i] * c[-1], side="right")), len(w) - 1)
        got.append(w[back][at] / math.fsum(w))
    return [None, torch.tensor(got, dtype=torch.float64)]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return _turned(s["x"], s["pos"], s["freq"], s["scale"], case["rot"], case["layout"])
    if kind == "sample":
        return _exact_sample(s)
    h, kv, d, page, w = case["heads"], case["kv"], case["d"], case["page"], case["window"]
    fresh, total = _lengths(case)
    if kind == "append":
        pos = torch.cat([torch.arange(t - f, t, device=DEV) for f, t in zip(fresh, total)])
        x = s["qkv"].view(-1, h + 2 * kv, d)
        q, k = _turned(x[:, :h], pos, s["freq"], s["scale"], d, "half"), _turned(x[:, h:h + kv], pos, s["freq"], s["scale"], d, "half")
        v = x[:, h + kv:].double()
        if case["int8"]:
            (ck, sk), (cv, sv) = _codes(k), _codes(v)
            k, v = ck * sk[..., None], cv * sv[..., None]
        return [q, k, v]
    out, at = torch.zeros((s["rows"], h, d), dtype=torch.float64, device=DEV), 0
    for i, (f, t) in enumerate(zip(fresh, total)):
        if not f:
            continue
        lo = max(0, t - f + 1 - w) // page if w else 0
        pages = s["table"][i, lo:-(-t // page)].long()
        q = s["q"][at:at + f].double()
        pos, key = torch.arange(t - f, t, device=DEV)[:, None], torch.arange(lo * page, t, device=DEV)
        hide = (key > pos) | (key <= pos - w) if w else key > pos
        for j in range(kv):
            k, v = (s[c][pages, j].double() * (s["s" + c][pages, j].double()[..., None] if case["int8"] else 1.0) for c in "kv")
            k, v = k.reshape(-1, d)[:len(key)], v.reshape(-1, d)[:len(key)]
            for head in range(j * h // kv, (j + 1) * h // kv):
                a = torch.softmax((q[:, head] @ k.t() / math.sqrt(d)).masked_fill_(hide, -math.inf), 1)
                out[at:at + f, head] = a @ v
        at += f
    return out
