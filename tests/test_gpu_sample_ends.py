"""Sampling where rows reach beyond the bins that the kernels count logits in:
tokens far below the largest logit that are still likely, prefixes that end among
very many small weights."""

import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import serving
from serving import DEV
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


@pytest.mark.parametrize("dt,low,t", [(torch.float32, -27.75, 1.0), (torch.bfloat16, -27.75, 1.0),
                                      (torch.bfloat16, -0.0625, 0.0625 / 27.75), (torch.float32, -0.0625, 0.0625 / 27.75)])
@pytest.mark.parametrize("n", [1 << 24, 1 << 21])
def test_nucleus_that_ends_among_millions_of_small_weights(n, dt, low, t):
    """One likely token at the end, n - 1 equal ones of weight w = 2^-40 before it, and a
    top_p whose goal lies among them: kept are the largest and the first
    ceil((top_p Z - 1) / w) of the others, exactly.  Drawn is number floor(u Zk / w).

    u is taken for the middle between two tokens; as binary32 it is within 2^-24 of
    that, 0.06 tokens at a million of them.  w is within 2^-50 of itself, and sums of
    n terms within n 2^-53 (2^-29): the tokens' numbers by less than 0.01."""
    t = float(np.float32(t))
    w = Fraction(math.exp(low / t))
    z = 1 + (n - 1) * w
    p = np.float32(1 - float((n - 1) * w) * 0.6)  # the goal: 40 of 100 small ones
    kept = math.ceil((Fraction(float(p)) * z - 1) / w)
    assert 0.1 * n < kept < 0.9 * n
    zk = 1 + kept * w
    want = [0, 5, 1000, min(1000000, kept // 2)]
    u = [float((Fraction(2 * i + 1, 2)) * w / zk) for i in want]
    # near the border, where a few tokens more or less do not count: kept, and not kept
    u += [float(kept * Fraction(99, 100) * w / zk), float(kept * Fraction(101, 100) * w / zk), 0.5]
    l = torch.full((1, n), low, dtype=dt, device=DEV)
    l[0, n - 1] = 0.0
    l = l.expand(len(u), n).contiguous()
    token, prob = w8a8.sample(l, torch.tensor(u, device=DEV), t, 0, float(p))
    token, prob = token.tolist(), prob.double().tolist()
    assert token[:4] == want
    assert abs(token[4] - 0.99 * kept) < 1e-4 * kept and token[5:] == [n - 1, n - 1]
    # kept is off by n 2^-53 / w tokens at the most, where sums round
    slack = 2.0 ** -24 + 2.0 ** -40 + n * 2.0 ** -53
    for i, x in zip(token, prob):
        exact = float((w if i < n - 1 else 1) / zk)
        assert abs(x - exact) <= slack * exact


def masked(rows, n, allowed, dt, seed, low=-math.inf):
    """Rows of which all but `allowed` logits are `low`."""
    g = serving.gen(seed)
    l = torch.full((rows, n), low)
    for i in range(rows):
        at = torch.randperm(n, generator=g)[:allowed]
        l[i, at] = torch.randn(allowed, generator=g) * 3
    return l.to(dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("low", [-math.inf, math.nan, -3e38, -1e4])
def test_masked_rows(dt, low):
    """Fewer logits than top_k that can be drawn, with every other filter; and the
    same with values far below in their place, which count among the top_k."""
    for n, allowed in ((50, 3), (9000, 20), (40001, 49), (40001, 1)):
        l, u = masked(6, n, allowed, dt, n, low), uniform(6, n)
        for a in (dict(k=50), dict(k=50, p=0.9), dict(k=n - 1), dict(k=n - 1, p=0.999999, t=2.0), dict(k=50, m=0.01),
                  dict(k=50, m=1e-30), dict(k=50, p=0.8, m=0.05), dict(k=50, t=1e4), dict(k=50, t=1e4, m=0.5), dict(k=1)):
            check(l, u, **a)
    l[:, ::2] = -math.inf  # far values beside masked ones: kept up to the 50th
    check(l, uniform(6, 5), k=50, t=1e4)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("low", [-math.inf, -3e38])
def test_masked_rows_take_about_as_long_as_others(dt, low):
    """Both in the same two launches: four times the time leaves room for the look at
    the rest of the row, passes over the row would take about twenty times."""
    def ms(l):
        u = torch.full((l.shape[0],), 0.5, device=DEV)
        run = lambda: w8a8.sample(l, u, 1.0, 50, 0.9)
        run()
        best = math.inf
        for _ in range(5):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            for _ in range(5):
                run()
            e[1].record()
            torch.cuda.synchronize()
            best = min(best, e[0].elapsed_time(e[1]))
        return best

    l = torch.randn((64, 262144), generator=serving.gen(1)).to(dt).to(DEV)
    m = torch.full_like(l, low)
    m[:, 777:797] = l[:, 777:797]
    assert ms(m) <= 4 * ms(l)


def test_signalling_nan_logits():
    """NaN of any bits are never drawn and hide no other logit."""
    g = serving.gen(1)
    l = torch.randn((4, 9000), generator=g).to(torch.bfloat16)
    u = uniform(4)
    bits = l.view(torch.int16)
    bits[:, ::7], bits[:, 1::7], bits[:, 2::7] = 0x7f81, 0xff81 - 65536, 0x7fc0
    wide = l.view(torch.int16).int() << 16
    wide[:, 3::7] = 0x7f800001
    quiet = lambda x: torch.where(x.isnan(), torch.tensor(math.nan, dtype=x.dtype), x)
    for x in (l, wide.view(torch.float32)):
        for a in ({}, dict(t=0.0), dict(k=40), dict(p=0.9), dict(m=0.1), dict(k=8000, p=0.999), dict(t=100.0)):
            want = check(quiet(x), u, **a)
            t, k, p, m = (a.get(c, d) for c, d in (("t", 1.0), ("k", 0), ("p", 1.0), ("m", 0.0)))
            assert torch.equal(w8a8.sample(x.to(DEV), u.to(DEV), t, k, p, m)[0], want), a
