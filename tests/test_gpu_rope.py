"""Rotary positions and the paged cache's append on the GPU against the plain
binary64 forms of tests/serving.py."""

import sys

import numpy as np
import pytest
import torch

import serving
from serving import DEV, Paged
from paper_2608_28003_amd import w8a8

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def make_rope(d, rot, layout, scaling="none", device=DEV):
    return w8a8.Rope.make(d, rot, 1e4, layout, scaling, 1.0 if scaling == "none" else 8.0, 4096, device)


def off(out, want, slack, dt):
    """The share of the bound used: the rotation's slack, then one rounding."""
    half = torch.finfo(dt).eps / 2
    bound = (want.abs() + slack) * half + slack + 1e-300
    return float(((out.double() - want).abs() / bound).max())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,d,rot,scaling", [
    (1, 1, 16, 16, "none"), (1, 5, 256, 256, "linear"), (7, 3, 80, 32, "yarn"), (65, 18, 128, 64, "ntk"),
    (33, 2, 96, 96, "none"), (5, 1, 1024, 512, "yarn"), (130, 4, 256, 64, "none"), (2, 70, 128, 128, "linear")])
def test_rope(rows, heads, d, rot, scaling, layout, dt):
    g = serving.gen(rows + d)
    x = (torch.randn((rows, heads, d), generator=g) * 3).to(dt)
    pos = torch.randint(0, 1 << 20, (rows,), generator=g, dtype=torch.int32)
    r = make_rope(d, rot, layout, scaling)
    want = serving.turned(x.double(), pos, r.freq.cpu(), r.scale, rot, layout)
    slack = serving.turn_slack(x.double(), r.scale, rot, layout)
    slack[..., rot:] = 0
    # rows inside a wider row, and behind them what must stay
    wide = torch.full((rows, heads * d + 24), 7.0, dtype=dt, device=DEV)
    wide[:, :heads * d] = x.reshape(rows, -1).to(DEV)
    view = wide[:, :heads * d].view(rows, heads, d) if rows == 1 else wide.as_strided((rows, heads, d), (heads * d + 24, d, 1))
    out = w8a8.rope(r, view, pos.to(DEV))
    used = off(out.cpu(), want, slack, dt)
    same = w8a8.rope(r, view, pos.to(DEV), out=view)
    say("  rope: %.3f of the bound" % used)
    assert used <= 1
    assert same is view and torch.equal(view, out)
    assert (wide[:, heads * d:] == 7.0).all()


def test_far_positions_keep_their_angles():
    """At position 2^30 a binary32 angle would be off by tens of radians."""
    r = make_rope(128, 128, "half")
    pos = torch.tensor([2 ** 30 - 1, 2 ** 31 - 1, 0, 1], dtype=torch.int32)
    x = torch.randn((4, 2, 128), generator=serving.gen(5))
    want = serving.turned(x.double(), pos, r.freq.cpu(), r.scale, 128, "half")
    # the binary64 product pos * freq rounds at 2^-53 of up to 2^31 radians, here and in the reference
    slack = serving.turn_slack(x.double(), 1.0, 128, "half") * (1 + 2.0 ** 31 * 2.0 ** -53 * 2.0 ** 23)
    assert off(w8a8.rope(r, x.to(DEV), pos.to(DEV)).cpu(), want, slack, torch.float32) <= 1


def test_position_zero_is_the_identity():
    x = torch.randn((3, 2, 256), generator=serving.gen(1)).to(torch.bfloat16).to(DEV)
    out = w8a8.rope(make_rope(256, 256, "half"), x, torch.zeros(3, dtype=torch.int32, device=DEV))
    assert torch.equal(out, x)


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("fresh,ctx,heads,n_kv,d,page,rot", [
    ([1], [1], 4, 1, 256, 16, 256), ([1, 1, 1], [40, 7, 129], 4, 1, 256, 64, 256), ([5, 0, 17], [5, 30, 40], 8, 4, 256, 16, 128),
    ([33, 2], [100, 2], 6, 2, 128, 32, 64), ([0, 3, 0, 0, 70, 0], [4, 3, 1, 9, 90, 2], 16, 8, 128, 128, 128)])
def test_append(fresh, ctx, heads, n_kv, d, page, rot, layout, int8):
    h = Paged(fresh, ctx, n_kv, d, page, int8, seed=3)
    g = serving.gen(11)
    pad, width = 2, (heads + 2 * n_kv) * d
    qkv = (torch.randn((h.rows + pad, width), generator=g) * 2).to(torch.bfloat16)
    if h.rows > 1:
        qkv[1, heads * d:(heads + 1) * d] = 0  # a key of zeros: scale 0, codes 0
    r = make_rope(d, rot, layout)
    cache, batch = h.cache(w8a8), h.batch(w8a8)
    before = [t.clone() for t in (cache.k, cache.v)] + ([cache.sk.clone(), cache.sv.clone()] if int8 else [])
    dev = qkv.to(DEV)
    out = torch.full((h.rows + pad, heads, d), 5.0, dtype=torch.bfloat16, device=DEV)
    w8a8.kv_append(dev, cache, batch, heads, rope=r, out=out)
    k_read, v_read = (torch.full((h.rows + pad, n_kv, d), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    w8a8.kv_read(cache, batch, h.rows + pad, k_read, v_read)

    pos = h.positions()
    x = qkv[:h.rows].double().view(h.rows, heads + 2 * n_kv, d)
    want = serving.turned(x[:, :heads + n_kv], pos, r.freq.cpu(), r.scale, rot, layout)
    slack = serving.turn_slack(x[:, :heads + n_kv], r.scale, rot, layout)
    slack[..., rot:] = 0
    assert off(out[:h.rows].cpu(), want[:, :heads], slack[:, :heads], torch.bfloat16) <= 1
    assert (out[h.rows:] == 5.0).all() and (k_read[h.rows:] == 5.0).all() and (v_read[h.rows:] == 5.0).all()
    wk, sk64, v = want[:, heads:], slack[:, heads:], x[:, heads + n_kv:]
    row = 0
    touched = torch.zeros(before[0].shape[:3], dtype=torch.bool)
    for s, (f, c) in enumerate(zip(fresh, ctx)):
        for t in range(f):
            p = c - f + t
            pg, slot = int(h.table[s, p // page]), p % page
            touched[pg, :, slot] = True
            ck, cv = cache.k[pg, :, slot].cpu(), cache.v[pg, :, slot].cpu()
            if int8:
                a, b = cache.sk[pg, :, slot].cpu().double(), cache.sv[pg, :, slot].cpu().double()
                top = wk[row].abs().amax(-1)
                assert ((a - top / 127).abs() <= (sk64[row].amax(-1) + top * 2.0 ** -23) / 127).all()
                # half a step of the code, the rotation's slack, and v / s rounded near a half
                bound = a[:, None] * (0.5 + 127 * 2.0 ** -23) + sk64[row]
                assert ((ck.double() * a[:, None] - wk[row]).abs() <= bound).all()
                qv, sv = serving.codes_of(v[row].float().numpy())
                assert np.array_equal(cv.numpy(), qv) and np.array_equal(b.float().numpy(), sv)
                assert torch.equal(k_read[row].cpu(), (ck.float() * a.float()[:, None]).to(torch.bfloat16))
                assert torch.equal(v_read[row].cpu(), (cv.float() * b.float()[:, None]).to(torch.bfloat16))
            else:
                assert off(ck, wk[row], sk64[row], torch.bfloat16) <= 1
                assert torch.equal(cv.double(), v[row])
                assert torch.equal(k_read[row].cpu(), ck) and torch.equal(v_read[row].cpu(), cv)
            row += 1
    for t, old in zip([cache.k, cache.v] + ([cache.sk, cache.sv] if int8 else []), before):
        same = (t == old) | (t.isnan() & old.isnan()) if t.is_floating_point() else t == old
        assert same[~touched].all()  # nothing but the new rows is written
    # in place: the queries over themselves in the projection's rows
    q = dev.as_strided((h.rows + pad, heads, d), (width, d, 1))
    tail = dev[:, heads * d:].clone()
    w8a8.kv_append(dev, cache, batch, heads, rope=r, out=q)
    assert torch.equal(q[:h.rows], out[:h.rows]) and torch.equal(dev[:, heads * d:], tail)
    assert torch.equal(q[h.rows:].cpu().reshape(pad, -1), qkv[h.rows:, :heads * d])


@pytest.mark.parametrize("int8", [True, False])
def test_append_without_rotation_and_without_pages(int8):
    """rope None; a hole in the table, a position beyond the table and a context
    shorter than its new tokens store nothing; reads there give zeros."""
    h = Paged([4, 3, 4], [40, 3, 20], 1, 256, 16, int8, seed=8, holes={(0, 2)})
    qkv = torch.randn((11, 1536), generator=serving.gen(2)).to(torch.bfloat16).to(DEV)
    cache = h.cache(w8a8)
    b = h.batch(w8a8)
    b.ctx_len = torch.tensor([40, 2, 50], dtype=torch.int32, device=DEV)  # second: a position of -1; third: 46 .. 49, table ends at 48
    old = cache.k.clone()
    q = w8a8.kv_append(qkv, cache, b, 4)
    assert torch.equal(q.view(11, -1), qkv[:, :1024])
    k, v = w8a8.kv_read(cache, b, 11)
    # 36 .. 39 lie in the hole (page 2); third: page 2 is not in its table either
    assert (k[:4] == 0).all() and (v[:4] == 0).all() and (k[4] == 0).all() and (k[7:] == 0).all()
    assert (k[5:7] != 0).any(-1).all() and (v[5:7] != 0).any(-1).all()
    changed = [i for i in range(old.shape[0]) if not torch.equal(torch.nan_to_num(cache.k[i].float()), torch.nan_to_num(old[i].float()))]
    assert changed == [int(h.table[1, 0])]


def test_binding_refusals():
    r = make_rope(256, 256, "half")
    x = torch.zeros((4, 5, 256), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(4, dtype=torch.int32, device=DEV)
    for bad in (dict(x=x.transpose(0, 1)), dict(pos=pos.long()), dict(pos=pos[:3]), dict(x=x[..., :128]), dict(x=x.cpu()),
                dict(out=x.float()), dict(r=w8a8.Rope(256, 256, "other", r.freq)), dict(r=w8a8.Rope(256, 256, "half", r.freq.float())),
                dict(r=w8a8.Rope(256, 128, "half", r.freq))):
        a = dict(r=r, x=x, pos=pos)
        a.update(bad)
        with pytest.raises(ValueError):
            w8a8.rope(**a)
    h = Paged([4], [4], 1, 256, 16, True)
    cache, b = h.cache(w8a8), h.batch(w8a8)
    qkv = torch.zeros((4, 1536), dtype=torch.bfloat16, device=DEV)
    for bad in (dict(qkv=qkv.float()), dict(n_heads=5), dict(cache=w8a8.PagedKV(cache.k, cache.v)),
                dict(cache=w8a8.PagedKV(cache.k, cache.v, cache.sk)), dict(cache=w8a8.PagedKV(cache.k, cache.v[:1], cache.sk, cache.sv)),
                dict(batch=w8a8.PagedBatch(b.table.long(), b.q_start, b.ctx_len, 4)),
                dict(batch=w8a8.PagedBatch(b.table, b.q_start[:1], b.ctx_len, 4)), dict(out=qkv)):
        a = dict(qkv=qkv, cache=cache, batch=b, n_heads=4)
        a.update(bad)
        with pytest.raises(ValueError):
            w8a8.kv_append(**a)
    with pytest.raises(ValueError):
        w8a8.attn_paged(torch.zeros((4, 4, 128), dtype=torch.bfloat16, device=DEV), cache, b)
    with pytest.raises(w8a8.W8A8Error):
        w8a8.attn_paged(torch.zeros((4, 4, 256), dtype=torch.bfloat16, device=DEV), cache, b, window=0)
