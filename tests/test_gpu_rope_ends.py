"""Appending rows to a paged cache whose values are not ordinary numbers."""

import math

import pytest
import torch

import serving
from serving import DEV
from paper_2608_28003_amd import w8a8

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def test_append_quantises_as_the_contiguous_cache():
    """Without a rotation an INT8 cache gets the codes and scales of kv_quantize,
    bit for bit: rows of all magnitudes, of zeros, with infinities and NaN, of NaN alone."""
    g, n, nan, inf = serving.gen(1), 512, math.nan, math.inf
    x = (torch.randn((n, 256), generator=g) * torch.exp(torch.randn((n, 1), generator=g) * 20)).to(torch.bfloat16)
    x[3], x[4, 5], x[5, 7], x[6], x[7], x[8, ::2] = 0.0, inf, nan, nan, 1e-40, -inf
    x[9], x[10, 0], x[10, 1:], x[11, :255], x[12] = torch.finfo(torch.bfloat16).max, 9.2e-41, 0.0, nan, inf
    codes, scales = w8a8.kv_quantize(x.to(DEV))
    assert scales[6].isnan()
    cache = w8a8.PagedKV.empty(n // 16, 16)
    qkv = torch.cat([torch.zeros((n, 1024), dtype=torch.bfloat16), x, x], 1).to(DEV)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    w8a8.kv_append(qkv, cache, w8a8.PagedBatch(torch.arange(n // 16, dtype=torch.int32, device=DEV)[None].contiguous(),
                                               ints(0, n), ints(n), n), 4)
    for c, s in ((cache.k, cache.sk), (cache.v, cache.sv)):
        s = s.view(-1)
        assert torch.equal(c.view(-1, 256), codes)
        assert ((s == scales) | (s.isnan() & scales.isnan())).all()
