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
