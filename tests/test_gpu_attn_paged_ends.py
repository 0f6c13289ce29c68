"""Attention over a paged cache at the ends of its ranges."""

import pytest
import torch

import serving
from serving import DEV
from paper_2608_28003_amd import w8a8
from test_gpu_attn_paged import attend

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("int8", [True, False])
def test_context_beyond_the_largest_table(int8):
    """A table of 2^30 positions, mostly not held, and tiles in one piece of that
    length: a context beyond it gives zeros at once, the sequence beside it its
    attention."""
    page, group, fresh = 65536, 64, [20, 490]
    g = serving.gen(3)
    cache = w8a8.PagedKV.empty(2, page, head_dim=128, int8=int8)
    kv = [torch.randn((490, 128), generator=g) for _ in range(2)]
    if int8:
        for (x, pool, scale) in ((kv[0], cache.k, cache.sk), (kv[1], cache.v, cache.sv)):
            c, s = serving.codes_of(x.numpy())
            pool[1, 0, :490], scale[1, 0, :490] = torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV)
    else:
        cache.k[1, 0, :490], cache.v[1, 0, :490] = (x.to(torch.bfloat16).to(DEV) for x in kv)
    q = torch.randn((510, group, 128), generator=g).to(torch.bfloat16).to(DEV)
    start = torch.tensor([0, 20, 510], dtype=torch.int32, device=DEV)
    table = torch.full((2, (1 << 30) // page), -1, dtype=torch.int32, device=DEV)
    table[1, 0] = 1
    ctx = torch.tensor([2 ** 31 - 1, 490], dtype=torch.int32, device=DEV)
    out = w8a8.attn_paged(q, cache, w8a8.PagedBatch(table, start, ctx, 490))
    assert (out[:20] == 0).all()
    one = w8a8.PagedBatch(table[1:, :1].contiguous(), start[1:] - 20, ctx[1:], 490)
    want = w8a8.attn_paged(q[20:], cache, one)
    # the same tiles, perhaps in other pieces: each within half a step of bf16 and the
    # weights' rounding (2^-8 of the mean of |v|, at most max |v|) of the other
    top = 2 * 2.0 ** -8 * max(float(x.abs().max()) for x in kv)
    assert ((out[20:].double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs() + top).all()
    assert (out[20:] != 0).any(-1).all()


@pytest.mark.parametrize("int8", [True, False])
def test_a_scale_of_zero_weighs_all_keys_alike(int8):
    """... however large the scores are; and one below the normal range as well.

    Queries of 5e35 against rows of 128 values of size 1.5, three of them three times that:
    products add up to 5e35 * 1.5 * 11 = 1e37, a thirtieth of what binary32 holds.  The sums
    over INT8 rows are of codes, up to 16 to 20 times their values: a tenth as large there."""
    large = 5e34 if int8 else 5e35
    h = serving.Paged([40, 1, 3], [90, 70, 3], 2, 128, 16, int8, seed=9)
    attend(h, 4, scale=0.0, q_scale=large)
    attend(h, 4, scale=-0.0, q_scale=large)
    attend(h, 4, scale=1e-40)
    attend(h, 4, scale=-1e-40, q_scale=large)


def check_rows(out, ref, keys, d):
    """As serving.check_attention, element by element, for sequences of at most 16 rows:
    their weights go into the products as two bf16 values, the second one the first one's
    rounding error (half a step of it, 2^-8) within half a step: 2^-16 of sum p |v|."""
    want, wide, _, top = ref
    slack = (2 * (d + 8) * 2.0 ** -24 * top[..., None] + 2.0 ** -19 + 2 * keys * 2.0 ** -24) * wide
    bound = 2.0 ** -8 * want.abs() * (1 + 2.0 ** -7) + 2.0 ** -16 * wide + slack
    err = (out.double() - want).abs()
    assert (err <= bound).all(), "%g of the bound" % float((err / bound.clamp_min(1e-300)).max())


@pytest.mark.parametrize("int8", [True, False])
@pytest.mark.parametrize("d,heads", [(128, 8), (256, 4)])
def test_weights_of_few_rows_have_sixteen_bits(d, heads, int8):
    """Few keys and small scores, so that one bf16 value a weight would show."""
    for seed, (fresh, ctx) in enumerate((([1, 1, 1], [5, 17, 40]), ([2, 1], [9, 33]), ([1], [3]))):
        h = serving.Paged(fresh, ctx, 2, d, 16, int8, seed=seed)
        q = (torch.randn((h.rows, heads, d), generator=serving.gen(seed)) * 0.05).to(torch.bfloat16)
        out = w8a8.attn_paged(q.to(DEV), h.cache(w8a8), h.batch(w8a8))
        check_rows(out.cpu(), h.attend(q, 2 ** 31 - 1, d ** -0.5), max(ctx), d)


@pytest.mark.parametrize("int8", [True, False])
def test_a_prompt_in_chunks_attends_alike(int8):
    """Three prompts at once (tiles), in chunks and token by token (rows): each
    one's last token attends alike.

    Two results differ by their own rounding (half a step each, 2^-8 of each), by
    the weights' (2^-8 of sum p |v| in tiles, 2^-16 in rows) and by the binary32 sums, as
    in serving.check_attention; sum p |v| is at most the largest |v|, a score's sum
    |q| |k| at most the norms' product."""
    lens, page, heads, window = [37, 64, 5], 16, 4, 50
    g = serving.gen(7)
    qkv = [torch.randn((n, (heads + 2) * 256), generator=g).to(torch.bfloat16).to(DEV) for n in lens]
    table = torch.randperm(24, generator=g).int().view(3, 8).to(DEV)
    rope = w8a8.Rope.make(256)

    def batch(fresh, done):
        start = torch.tensor([0] + fresh, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(DEV)
        return w8a8.PagedBatch(table, start, torch.tensor(done, dtype=torch.int32, device=DEV), max(fresh))

    def feed(part):
        cache, done, last = w8a8.PagedKV.empty(24, page, int8=int8), [0, 0, 0], [None] * 3
        while done != lens:
            fresh = [min(part, n - x) for n, x in zip(lens, done)]
            rows = torch.cat([x[a:a + f] for x, a, f in zip(qkv, done, fresh)])
            done = [a + f for a, f in zip(done, fresh)]
            b = batch(fresh, done)
            q = w8a8.kv_append(rows, cache, b, heads, rope=rope)
            out = w8a8.attn_paged(q, cache, b, window=window)
            for s, f in enumerate(fresh):
                if f:
                    last[s] = (out[sum(fresh[:s + 1]) - 1].double(), q[sum(fresh[:s + 1]) - 1].double())
        return cache, last

    cache, whole = feed(64)
    k, v = (x.double() for x in w8a8.kv_read(cache, batch(lens, lens), sum(lens)))
    for part in (32, 3, 1):
        _, parts = feed(part)
        at = 0
        for n, (a, q), (b, _) in zip(lens, whole, parts):
            rows = slice(at + max(0, n - window), at + n)
            at += n
            wide = v[rows, 0].abs().amax(0)
            top = float(q.norm(dim=-1).max() * k[rows, 0].norm(dim=-1).max()) / 16
            slack = 2 * (2 * 264 * 2.0 ** -24 * top + 2.0 ** -19 + 2 * n * 2.0 ** -24)
            bound = 2.0 ** -8 * (a.abs() + b.abs()) * (1 + 2.0 ** -7) + (2 * 2.0 ** -8 + slack) * wide
            assert ((a - b).abs() <= bound).all(), (part, float(((a - b).abs() / bound).max()))
            assert (a != 0).any(-1).all()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("fresh,heads", [(40, 2), (200, 4), (3, 2)])
def test_scales_that_are_nan_stay_with_the_tokens_that_attend_them(fresh, heads, d):
    """INT8: a NaN scale of a key or value reaches the tokens that attend the row, whose
    results are NaN, and no other: earlier tokens, and later ones behind the window."""
    h = serving.Paged([fresh, 1], [fresh + 30, 9], 1, d, 16, True, seed=d)
    q = torch.randn((h.rows, heads, d), generator=serving.gen(2)).to(torch.bfloat16).to(DEV)
    b, window = h.batch(w8a8), 25
    good = w8a8.attn_paged(q, h.cache(w8a8), b, window=window)
    at = fresh + 30 - 1 - fresh // 3  # a position among the new tokens
    page, slot = int(h.table[0, at // 16]), at % 16
    pos = torch.arange(30, fresh + 30)
    sees = (pos >= at) & (pos < at + window)
    for name in ("sk", "sv"):
        cache = h.cache(w8a8)
        getattr(cache, name)[page, 0, slot] = float("nan")
        out = w8a8.attn_paged(q, cache, b, window=window)
        assert out[:fresh][sees.to(DEV)].isnan().all()
        assert torch.equal(out[:fresh][~sees.to(DEV)], good[:fresh][~sees.to(DEV)]) and torch.equal(out[fresh:], good[fresh:])
