"""Attention of new tokens over a paged cache against the plain binary64 form
of tests/serving.py.  Unused slots of the cache hold NaN throughout."""

import sys

import pytest
import torch

import serving
from serving import DEV, Paged, check_attention
from paper_2608_28003_amd import w8a8

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

NONE = 2 ** 31 - 1


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def attend(h, heads, window=None, scale=None, pad=2, seed=4, q_scale=1.0):
    q = (torch.randn((h.rows + pad, heads, h.d), generator=serving.gen(seed)) * q_scale).to(torch.bfloat16)
    out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device=DEV)
    w8a8.attn_paged(q.to(DEV), h.cache(w8a8), h.batch(w8a8), window=window, scale=scale, out=out)
    assert (out[h.rows:] == 3.0).all()  # rows behind the last sequence
    ref = h.attend(q[:h.rows], NONE if window is None else window, h.d ** -0.5 if scale is None else scale)
    check_attention(out[:h.rows].cpu(), ref, max(h.ctx), h.d, "attention")
    return out, ref


CASES = [
    # new tokens, contexts, query heads, key/value heads, width, page, window
    ([1], [1], 4, 1, 256, 16, None),
    ([1], [31], 1, 1, 256, 16, None),
    ([1, 1, 1, 1], [5, 700, 64, 129], 4, 1, 256, 64, None),
    ([4, 1, 3], [300, 33, 3], 4, 1, 256, 32, None),
    ([4, 0, 5], [300, 9, 80], 8, 4, 256, 16, 40),
    ([33, 17, 1], [33, 100, 200], 4, 1, 256, 16, None),
    ([70, 3, 0, 129], [150, 3, 4, 129], 6, 2, 128, 32, None),
    ([40, 1], [300, 260], 16, 8, 128, 128, 7),
    ([65], [65], 5, 1, 128, 16, 1),
    ([260], [500], 2, 2, 256, 64, 100),
    ([20], [20], 24, 1, 128, 16, None),
    ([100, 31, 1], [1200, 31, 1100], 8, 1, 128, 16, None),
]


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("fresh,ctx,heads,n_kv,d,page,window", CASES)
def test_attention(fresh, ctx, heads, n_kv, d, page, window, int8):
    attend(Paged(fresh, ctx, n_kv, d, page, int8, seed=len(fresh)), heads, window)


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("fresh,ctx", [([1, 2], [3000, 2500]), ([40], [2100])])
def test_long_contexts(fresh, ctx, int8):
    """Long enough for several workgroups to share a row's keys."""
    attend(Paged(fresh, ctx, 1, 256, 64, int8, seed=6), 4)


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("fresh", [1, 50])
def test_holes_and_rows_without_keys(fresh, int8):
    """Pages that the table does not hold are skipped; a token whose whole
    window lies in them gets zeros, also where more than one workgroup looks."""
    for ctx, holes, window in ((200, {0, 3, 7}, None), (200, set(range(13)), None), (200, {11, 12}, 9), (1500, set(range(60)), None)):
        h = Paged([fresh, 1], [ctx, 40], 1, 256, 16, int8, seed=ctx, holes={(0, i) for i in holes})
        out, ref = attend(h, 4, window)
        empty = (ref[1] == 0).all(-1)
        assert (out[:h.rows].cpu()[empty] == 0).all()
        if len(holes) == 13:
            assert empty[:fresh].all()


def test_context_shorter_than_its_new_tokens():
    """Tokens before position 0 see nothing."""
    h = Paged([6], [6], 1, 128, 16, True)
    q = torch.randn((6, 2, 128), generator=serving.gen(1)).to(torch.bfloat16).to(DEV)
    b = h.batch(w8a8)
    b.ctx_len.fill_(2)
    out = w8a8.attn_paged(q, h.cache(w8a8), b)
    assert (out[:4] == 0).all() and (out[4:] != 0).any()
    for n in (0, -5, -2 ** 31):
        b.ctx_len.fill_(n)
        assert (w8a8.attn_paged(q, h.cache(w8a8), b) == 0).all()


@pytest.mark.parametrize("int8", [True, False])
def test_tables_that_lie(int8):
    """Entries outside the cache, a context beyond the table, rows beyond the
    call: nothing outside is read or written, and what is right stays right."""
    h = Paged([3, 2], [100, 50], 1, 256, 16, int8, seed=2, max_pages=8)
    q = torch.randn((5, 4, 256), generator=serving.gen(3)).to(torch.bfloat16).to(DEV)
    cache, b = h.cache(w8a8), h.batch(w8a8)
    good = w8a8.attn_paged(q, cache, b)
    b.table[0, 7] = 10 ** 9  # behind the context: never looked at
    assert torch.equal(w8a8.attn_paged(q, cache, b), good)
    b.table[0, :] = 10 ** 9
    out = w8a8.attn_paged(q, cache, b)
    assert (out[:3] == 0).all() and torch.equal(out[3:], good[3:])
    b.ctx_len[0] = 2 ** 31 - 1
    out = w8a8.attn_paged(q, cache, b)
    assert (out[:3] == 0).all() and torch.equal(out[3:], good[3:])
    b.q_start[2] = 7  # two rows more than there are: that sequence is left alone
    keep = torch.full_like(good, 2.0)
    w8a8.attn_paged(q, cache, b, out=keep)
    assert (keep[:3] == 0).all() and (keep[3:] == 2.0).all()


@pytest.mark.parametrize("int8", [True, False])
def test_scales_of_scores(int8):
    h = Paged([9, 1], [90, 70], 2, 128, 16, int8, seed=9)
    attend(h, 4, scale=0.0)
    attend(h, 4, scale=-0.05)
    attend(h, 4, scale=0.5, q_scale=2.0)  # one key takes nearly all


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("fresh", [2, 40])
def test_strides(fresh, int8):
    """Queries in the rows of a fused projection, results into wider rows."""
    h = Paged([fresh], [90], 1, 256, 32, int8, seed=5)
    qkv = torch.randn((fresh, 1536), generator=serving.gen(6)).to(torch.bfloat16)
    dev = qkv.to(DEV)
    wide = torch.full((fresh, 1104), 2.0, dtype=torch.bfloat16, device=DEV)
    w8a8.attn_paged(dev.as_strided((fresh, 4, 256), (1536, 256, 1)), h.cache(w8a8), h.batch(w8a8),
                    out=wide.as_strided((fresh, 4, 256), (1104, 256, 1)))
    ref = h.attend(qkv[:, :1024].reshape(fresh, 4, 256), NONE, 0.0625)
    check_attention(wide[:, :1024].cpu().reshape(fresh, 4, 256), ref, 90, 256, "strided")
    assert (wide[:, 1024:] == 2.0).all()


def test_many_sequences():
    """More sequences than lanes of a wave, some without new tokens."""
    fresh = [(3 * i) % 4 for i in range(150)]
    ctx = [f + (7 * i) % 40 + 1 for i, f in enumerate(fresh)]
    attend(Paged(fresh, ctx, 1, 128, 16, True, seed=1), 2)


def test_cache_beyond_32_bit_offsets():
    """A pool of more than 2^32 bytes a side; the sequence lives in its last pages."""
    n_pages = (1 << 32) // (64 * 512) + 9
    k = torch.zeros((n_pages, 1, 64, 256), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    small = Paged([20], [130], 1, 256, 64, False, seed=12)
    cache = w8a8.PagedKV(k, v)
    n = small.k.shape[0]
    k[-n:], v[-n:] = small.k.to(DEV), small.v.to(DEV)
    b = small.batch(w8a8)
    b.table += (n_pages - n) * (b.table >= 0).int()
    q = torch.randn((20, 4, 256), generator=serving.gen(13)).to(torch.bfloat16)
    out = w8a8.attn_paged(q.to(DEV), cache, b)
    check_attention(out.cpu(), small.attend(q, NONE, 0.0625), 130, 256, "far pages")
    one = w8a8.PagedBatch(b.table, torch.tensor([0, 1], dtype=torch.int32, device=DEV), b.ctx_len, 1)
    out = w8a8.attn_paged(q[:1].to(DEV), cache, one)
    small.fresh, small.rows = [1], 1
    check_attention(out.cpu(), small.attend(q[:1], NONE, 0.0625), 130, 256, "far pages, one token")


@pytest.mark.parametrize("int8", [True, False])
def test_one_token_agrees_with_the_contiguous_cache(int8):
    """A table that counts up is the contiguous cache of attn_decode."""
    t_max, pos = 1024, 777
    g = serving.gen(21)
    kv = [(torch.randn((t_max, 256), generator=g) * 2).to(torch.bfloat16).to(DEV) for _ in range(2)]
    row = (torch.randn(1536, generator=g) * 2).to(torch.bfloat16).to(DEV)
    flat = w8a8.KVCache(t_max, int8=int8)
    flat.fill(0, *kv)
    paged = w8a8.PagedKV.empty(t_max // 32, 32, int8=int8)
    for t, src in ((paged.k, flat.k), (paged.v, flat.v)) + (((paged.sk, flat.sk), (paged.sv, flat.sv)) if int8 else ()):
        t.view(-1).copy_(src.view(-1))
    b = w8a8.PagedBatch(torch.arange(t_max // 32, dtype=torch.int32, device=DEV)[None].contiguous(),
                        torch.tensor([0, 1], dtype=torch.int32, device=DEV),
                        torch.tensor([pos + 1], dtype=torch.int32, device=DEV), 1)
    for window in (t_max, 100):
        want = w8a8.attn_decode(row, flat, pos, window)
        q = w8a8.kv_append(row[None], paged, b, 4)
        out = w8a8.attn_paged(q, paged, b, window=window)
        assert torch.equal(paged.k.view(-1), flat.k.view(-1)) and torch.equal(paged.v.view(-1), flat.v.view(-1))
        # both within half a step of nearly the same binary32 result: at most one step apart
        a, c = out.view(-1).double(), want.double()
        assert ((a - c).abs() <= 2.0 ** -7 * c.abs() + 2.0 ** -16 * c.abs().max()).all()


@pytest.mark.parametrize("seqs,n_kv", [(70, 1), (130, 2), (200, 4), (300, 4), (513, 1), (520, 3)])
def test_contexts_of_many_lengths(seqs, n_kv):
    """A few long contexts among many short ones: sequences in one piece and in
    several, more of them than workgroups fit, and more than are shared out."""
    fresh = [(0 if i % 13 == 5 else 1 + i % 2) for i in range(seqs)]
    ctx = [f + (5 * i) % 60 + (2500 if i in (3, seqs - 2) else 0) for i, f in enumerate(fresh)]
    attend(Paged(fresh, ctx, n_kv, 128, 64, True, seed=seqs), n_kv)


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("window,holes", [(None, ()), (700, ()), (None, range(20, 60)), (300, range(40, 131))])
def test_tiles_in_pieces(d, int8, window, holes):
    """More than 16 rows over keys that several workgroups share, with a window and
    with pages given back."""
    h = Paged([45, 2], [2100, 1300], 2, d, 16, int8, seed=d, holes={(0, i) for i in holes})
    attend(h, 6, window)


@pytest.mark.parametrize("int8", [True, False])
def test_more_new_tokens_than_announced(int8):
    """A sequence of more new tokens than max_q is left alone; the others are not."""
    h = Paged([3, 40, 2], [50, 60, 70], 1, 128, 16, int8, seed=8)
    q = torch.randn((45, 2, 128), generator=serving.gen(9)).to(torch.bfloat16).to(DEV)
    good = w8a8.attn_paged(q, h.cache(w8a8), h.batch(w8a8))
    b = h.batch(w8a8)
    for max_q in (39, 3):
        b.max_q = max_q
        out = torch.full_like(q, 2.0)
        w8a8.attn_paged(q, h.cache(w8a8), b, out=out)
        assert (out[3:43] == 2.0).all()
        for s in (slice(0, 3), slice(43, 45)):  # cut into other pieces, perhaps
            assert (out[s].float() - good[s].float()).abs().max() <= 2.0 ** -7 * good.float().abs().max()


def test_workspace():
    h = Paged([1, 30], [600, 700], 1, 256, 64, True, seed=3)
    q = torch.randn((31, 4, 256), generator=serving.gen(3)).to(torch.bfloat16).to(DEV)
    cache, b = h.cache(w8a8), h.batch(w8a8)
    need = w8a8.attn_paged_workspace_bytes(31, 4, 1, 256, 2, b.max_q, b.table.shape[1] * 64)
    assert need > 0
    good = w8a8.attn_paged(q, cache, b)
    ws = torch.full((need + 256,), 0x7f, dtype=torch.uint8, device=DEV)
    assert torch.equal(w8a8.attn_paged(q, cache, b, ws=ws[:need]), good)
    assert (ws[need:] == 0x7f).all()
    with pytest.raises(w8a8.W8A8Error) as e:
        w8a8.attn_paged(q, cache, b, ws=ws[:need - 256])
    assert e.value.status == w8a8.EWORKSPACE
