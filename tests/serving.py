"""Plain binary64 forms of the serving operators (numpy / torch on the CPU), and
the inputs their tests share.  Written from the definitions in include/w8a8.h."""

import math

import numpy as np
import torch

DEV = "cuda:0"


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def turned(x, pos, freq, scale, rot, layout):
    """x: [rows, heads, d] float64; positions [rows]; one pair after the other."""
    out = x.clone()
    a = pos.double()[:, None] * freq
    c, s = torch.cos(a) * scale, torch.sin(a) * scale
    for j in range(rot // 2):
        i, k = (j, j + rot // 2) if layout == "half" else (2 * j, 2 * j + 1)
        out[..., i] = x[..., i] * c[:, j:j + 1] - x[..., k] * s[:, j:j + 1]
        out[..., k] = x[..., k] * c[:, j:j + 1] + x[..., i] * s[:, j:j + 1]
    return out


def turn_slack(x, scale, rot, layout):
    """What |a| + |b| of an element's pair, times scale, allows the binary32
    rotation to be off by, in units of 2^-21: the angle's fraction of a turn is
    rounded to binary32 (2 pi * 2^-26 in the angle), sine and cosine are within
    two steps of 2^-24, and the two products and their sum round once each."""
    x = x.abs()
    w = torch.zeros_like(x)
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    w[..., lo] = w[..., hi] = (x[..., lo] + x[..., hi]) * abs(scale)
    return w * 2.0 ** -21


def codes_of(x):
    """float32 rows -> (codes, scales) by the cache's rule, in binary32 steps."""
    x = np.asarray(x, np.float32)
    s = (np.abs(x).max(-1) / np.float32(127.0)).astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(s[..., None] > 0, x / s[..., None], np.float32(0.0))
    return np.clip(np.rint(q), -127, 127).astype(np.int8), s


class Paged:
    """A cache of random pages on the CPU, and the tables of sequences with
    given numbers of new tokens and contexts.  Slots that no position uses hold
    NaN (bf16) or NaN scales (INT8): they must never count."""

    def __init__(self, fresh, ctx, n_kv, d, page, int8, seed=0, holes=(), max_pages=None):
        g = gen(seed)
        self.fresh, self.ctx, self.n_kv, self.d, self.page, self.int8 = list(fresh), list(ctx), n_kv, d, page, int8
        blocks = [-(-c // page) for c in ctx]
        n = sum(blocks) + 2
        order = torch.randperm(n, generator=g)
        width = max_pages or max(1, max(blocks))
        self.table = torch.full((len(ctx), width), -1, dtype=torch.int32)
        at = 0
        for s, b in enumerate(blocks):
            for i in range(b):
                if (s, i) not in holes:
                    self.table[s, i] = int(order[at])
                at += 1
        x = [torch.randn((n, n_kv, page, d), generator=g) * 1.5 for _ in range(2)]
        for t in x:
            t[..., torch.randperm(d, generator=g)[:3]] *= 3.0
        used = torch.zeros((n, page), dtype=torch.bool)
        for s, c in enumerate(ctx):
            for i in range(blocks[s]):
                if self.table[s, i] >= 0:
                    used[self.table[s, i], :min(page, c - i * page)] = True
        if int8:
            (k, sk), (v, sv) = (codes_of(t.numpy()) for t in x)
            self.k, self.v, self.sk, self.sv = (torch.from_numpy(t) for t in (k, v, sk, sv))
            for t in (self.sk, self.sv):
                t.masked_fill_(~used[:, None], math.nan)
        else:
            self.k, self.v = (t.to(torch.bfloat16) for t in x)
            for t in (self.k, self.v):
                t.masked_fill_(~used[:, None, :, None], math.nan)
            self.sk = self.sv = None
        self.q_start = torch.tensor(np.cumsum([0] + list(fresh)), dtype=torch.int32)
        self.rows = int(sum(fresh))
        self.max_q = max(1, max(fresh))

    def cache(self, w8a8):
        dev = lambda t: None if t is None else t.to(DEV)
        return w8a8.PagedKV(dev(self.k), dev(self.v), dev(self.sk), dev(self.sv))

    def batch(self, w8a8):
        return w8a8.PagedBatch(self.table.to(DEV), self.q_start.to(DEV),
                               torch.tensor(self.ctx, dtype=torch.int32, device=DEV), self.max_q)

    def positions(self):
        return torch.cat([torch.arange(c - f, c) for f, c in zip(self.fresh, self.ctx)])

    def values(self, name, s, j):
        """(keys or values of sequence s, head j as float64 [ctx, d], held [ctx])."""
        pool, scale = getattr(self, name), getattr(self, "s" + name)
        out = torch.zeros((self.ctx[s], self.d), dtype=torch.float64)
        held = torch.zeros(self.ctx[s], dtype=torch.bool)
        for p in range(self.ctx[s]):
            page = int(self.table[s, p // self.page])
            if page >= 0:
                row = pool[page, j, p % self.page].double()
                out[p] = row if scale is None else row * scale[page, j, p % self.page].double()
                held[p] = True
        return out, held

    def attend(self, q, window, scale):
        """Per row and head: the result, sum p |v|, sqrt(sum p^2 v^2) (both over
        sum p) and the largest sum |q| |k| scale of a score; float64."""
        heads = q.shape[1]
        res = [torch.zeros(q.shape, dtype=torch.float64) for _ in range(3)] + [torch.zeros(q.shape[:2], dtype=torch.float64)]
        at = 0
        for s, (f, c) in enumerate(zip(self.fresh, self.ctx)):
            if f:
                pos, key = torch.arange(c - f, c)[:, None], torch.arange(c)
                for h in range(heads):
                    j = h // (heads // self.n_kv)
                    (k, held), (v, _) = self.values("k", s, j), self.values("v", s, j)
                    qq = q[at:at + f, h].double()
                    seen = (key <= pos) & held & (key > pos - window)
                    sc = (qq @ k.t() * scale).masked_fill(~seen, -math.inf)
                    m = sc.amax(1, keepdim=True)
                    p = torch.where(seen, torch.exp(sc - torch.where(m == -math.inf, 0.0, m)), 0.0)
                    den = p.sum(1, keepdim=True)
                    ok = den > 0
                    den = torch.where(ok, den, 1.0)
                    res[0][at:at + f, h] = p @ v / den
                    res[1][at:at + f, h] = p @ v.abs() / den
                    res[2][at:at + f, h] = ((p * p) @ (v * v)).sqrt() / den
                    res[3][at:at + f, h] = ((qq.abs() @ k.abs().t() * abs(scale)) * seen).amax(1)
            at += f
        return res


def check_attention(out, ref, keys, d, what):
    """out (bf16) against attend()'s results.

    Per element: half a bf16 step of the result (2^-8 |out|), the weights rounded
    to bf16 (2^-8 of sum p |v|), scores of d products summed in binary32 (each
    within (d + 8) 2^-24 of sum |q| |k|, twice for numerator and denominator), the
    exponential (2^-20 with the rounding of its argument, up to 64), and the binary32
    sums over the keys (keys * 2^-24, twice).  Over all elements the roundings of
    the weights are independent: their part is 2^-8 of sqrt(sum p^2 v^2), not of
    sum p |v|."""
    o = out.double()
    want, wide, rms, top = ref
    assert torch.isfinite(o).all(), what
    slack = (2 * (d + 8) * 2.0 ** -24 * top[..., None] + 2.0 ** -19 + 2 * keys * 2.0 ** -24) * wide
    err = (o - want).abs()
    bound = 2.0 ** -8 * want.abs() * (1 + 2.0 ** -7) + 2.0 ** -8 * wide + slack
    assert (err <= bound).all(), "%s: %g of the bound" % (what, float((err / bound.clamp_min(1e-300)).max()))
    total = 2.0 ** -8 * torch.linalg.norm(want) + 2.0 ** -8 * torch.linalg.norm(rms) + torch.linalg.norm(slack)
    assert torch.linalg.norm(o - want) <= total, "%s: %g of the norm's bound" % (what, float(torch.linalg.norm(o - want) / total))


def draw(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row, by the definition."""
    l = np.asarray(l, np.float64)
    l = np.where(np.isnan(l), -np.inf, l)
    top = l.max()
    if top == -np.inf:
        return -1, 0.0
    order = np.argsort(-l, kind="stable")
    if not temperature > 0:
        order, w = order[:1], np.ones(1)
    else:
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(l[order] == top, 1.0, np.exp((l[order] - top) / np.float64(temperature)))
        w = np.where((l[order] == -np.inf) | ((top == np.inf) & (l[order] != top)), 0.0, w)
        if 0 < top_k < len(w):
            w = w[:top_k]
        if top_p < 1:
            c = np.cumsum(w)
            w = w[:max(1, int((np.concatenate([[0.0], c[:-1]]) < max(0.0, np.float64(top_p)) * c[-1]).sum()))]
        if min_p > 0:
            w = w[:max(1, int((w >= np.float64(min_p)).sum()))]
        order = order[:len(w)]
    by = np.argsort(order)
    order, w = order[by], w[by]
    c = np.cumsum(w)
    hit = np.nonzero(c > np.float64(u) * c[-1])[0]
    at = int(hit[0]) if len(hit) else int(np.nonzero(w > 0)[0][-1])
    return int(order[at]), float(w[at] / c[-1])
