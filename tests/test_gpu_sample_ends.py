"""Sampling where rows reach beyond the bins that the kernels count logits in:
tokens far below the largest logit that are still likely."""

import math

import pytest
import torch

import serving
from paper_2608_28003_amd import w8a8
from test_gpu_sample import check, uniform

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_hot_rows_draw_from_all_their_logits(dt):
    """Logits more than 2047 values of 16 bits apart, at temperatures at which the
    farthest are drawn as well: without a filter, or with a top_k that keeps all."""
    u = torch.tensor([0.0, 0.2, 0.5, 0.8, 0.99, 1 - 2.0 ** -24])
    l = torch.full((6, 9), -100.0)
    l[:, 0] = 8.0
    for t in (5.0, 30.0, 1e3, math.inf):
        check(l.to(dt), u, t=t)
        check(l.to(dt), u, t=t, k=9)
    g = serving.gen(3)
    for n in (117, 8193, 40001):
        for sigma in (30.0, 1e3, 1e20):
            l = (torch.randn((6, n), generator=g) * sigma).to(dt)
            check(l, u, t=sigma)
            check(l, uniform(6, n), t=3.0 * sigma)
            check(l, uniform(6, n + 1), t=sigma, p=0.9)
            check(l, uniform(6, n + 2), t=sigma, m=0.2)
    l = (torch.randn((6, 20000), generator=g) * 50.0).to(dt)
    l[:, ::3] = -math.inf
    check(l, uniform(6), t=60.0)
