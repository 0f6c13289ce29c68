"""Sampling on the GPU against the plain binary64 form of tests/serving.py: the
tokens are equal, the probabilities within the rounding to binary32 (and the
sums' order, 2^-40 of it)."""

import math
import sys

import numpy as np
import pytest
import torch

import serving
from serving import DEV
from paper_2608_28003_amd import w8a8

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def check(logits, u, t=1.0, k=0, p=1.0, m=0.0, ld=None):
    """logits: CPU tensor [rows, n]; parameters: numbers or CPU tensors [rows]."""
    rows, n = logits.shape
    dev = logits.to(DEV)
    if ld is not None:
        wide = torch.full((rows, ld), 100.0, dtype=logits.dtype, device=DEV)
        wide[:, :n] = dev
        dev = wide[:, :n]
    put = lambda x: x.to(DEV) if isinstance(x, torch.Tensor) else x
    token, prob = w8a8.sample(dev, u.to(DEV), put(t), put(k), put(p), put(m))
    again, _ = w8a8.sample(dev, u.to(DEV), put(t), put(k), put(p), put(m))
    assert torch.equal(token, again)
    # a number goes through the call as binary32, so the definition gets that value, too
    at = lambda x, i, kind: kind(x[i]) if isinstance(x, torch.Tensor) else kind(np.float32(x))
    l = logits.float().numpy()
    for i in range(rows):
        want = serving.draw(l[i], float(u[i]), at(t, i, float), at(k, i, int), at(p, i, float), at(m, i, float))
        assert int(token[i]) == want[0], (i, int(token[i]), want)
        assert abs(float(prob[i]) - want[1]) <= (2.0 ** -24 + 2.0 ** -40) * want[1], (i, float(prob[i]), want)
    return token


def peaked(rows, n, dt, seed, sigma=2.5, top=9.0):
    g = serving.gen(seed)
    l = torch.randn((rows, n), generator=g) * sigma
    at = torch.randint(0, n, (rows, 20), generator=g)
    l.scatter_(1, at, top + 2.5 * torch.randn((rows, 20), generator=g))
    return l.to(dt)


def uniform(rows, seed=1):
    return torch.rand(rows, generator=serving.gen(seed))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 1000, 8191, 8192, 8193, 40001, 262144])
@pytest.mark.parametrize("mode", ["none", "k", "p", "m", "all", "greedy"])
def test_filters(mode, n, dt):
    rows = 3 if n > 100000 else 6
    l, g = peaked(rows, n, dt, n), serving.gen(n + 1)
    r = torch.rand((4, rows), generator=g)
    a = {"t": 0.5 + r[0]}
    if mode in ("k", "all"):
        a["k"] = (1 + 60 * r[1]).int()
    if mode in ("p", "all"):
        a["p"] = 0.3 + 0.69 * r[2]
    if mode in ("m", "all"):
        a["m"] = 0.2 * r[3]
    if mode == "greedy":
        a["t"] = torch.tensor([0.0, -1.0] * 3)[:rows]
    check(l, uniform(rows, n), **a)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_flat_logits(dt):
    """No token stands out: the nucleus is most of the vocabulary, and its border
    lies where bf16 logits are near 0 and finely spaced."""
    g = serving.gen(3)
    for sigma in (0.01, 1.0, 30.0):
        l = (torch.randn((4, 30011), generator=g) * sigma).to(dt)
        check(l, uniform(4), p=torch.tensor([0.1, 0.5, 0.9, 0.999]))
        check(l, uniform(4, 2), k=torch.tensor([1, 1000, 20000, 30011], dtype=torch.int32))
        check(l - 50.0, uniform(4, 3), t=3.0, p=0.7, k=15000)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_equal_logits(dt):
    """Ties: the lowest indexes stay."""
    for n in (5, 9000, 20000):
        l = torch.full((5, n), -3.0, dtype=dt)
        u = torch.tensor([0.0, 0.3, 0.5, 0.99, 1 - 2.0 ** -24])
        check(l, u)
        check(l, u, k=max(1, n // 3))
        check(l, u, p=0.4)
        check(l, u, k=max(1, n // 2), p=0.5, m=1.0)
        check(l, u, t=0.0)
    l = torch.zeros((2, 4000), dtype=dt)
    l[:, ::2] = -0.0  # equal to 0
    check(l, torch.tensor([0.2, 0.9]), k=10)
    l = torch.randint(0, 4, (6, 50000), generator=serving.gen(2)).to(dt)
    check(l, uniform(6), k=torch.tensor([5, 12000, 13000, 30000, 49999, 50000], dtype=torch.int32))
    check(l, uniform(6), p=torch.tensor([0.01, 0.2, 0.5, 0.65, 0.9, 0.99]))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_infinite_and_nan_logits(dt):
    inf, nan = math.inf, math.nan
    rows = [[-inf] * 6, [nan] * 6, [nan, -inf, nan, 1.0, -inf, nan], [inf, 1.0, inf, nan, -inf, 2.0], [inf] * 6, [0.0, -inf, 0.0, nan, 0.0, -inf],
            [-3e38, -3e38, 3e38, 0.0, 3e38, nan], [-inf, -inf, -1e30, -inf, -inf, -inf]]
    l = torch.tensor(rows).to(dt)
    for u in (0.0, 0.4, 0.999):
        uu = torch.full((len(rows),), u)
        for a in ({}, dict(k=2), dict(p=0.5), dict(m=0.5), dict(k=4, p=0.9, m=0.1), dict(t=0.0), dict(t=100.0), dict(t=1e-6), dict(k=6, p=0.999999)):
            t = check(l, uu, **a)
            assert int(t[0]) == -1 and int(t[1]) == -1 and int(t[2]) == 3


def test_parameters_at_their_ends():
    l = peaked(8, 5000, torch.bfloat16, 4)
    u = uniform(8)
    check(l, u, k=torch.tensor([-5, 0, 1, 4999, 5000, 5001, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32))
    check(l, u, p=torch.tensor([-1.0, 0.0, 1e-30, 1.0, 2.0, 0.9999999, math.inf, -math.inf]))
    check(l, u, m=torch.tensor([-1.0, 0.0, 1e-30, 1.0, 2.0, 0.9999999, math.inf, -math.inf]))
    check(l, torch.tensor([0.0, -1.0, 1.0, 2.0, 1 - 2.0 ** -24, 2.0 ** -149, math.inf, -math.inf]))
    # NaN: off, and a uniform number that is none draws the first token
    dev, ud = l.to(DEV), u.to(DEV)
    off = torch.full((8,), math.nan, device=DEV)
    assert torch.equal(w8a8.sample(dev, ud, 1.0, 0, off, off)[0], w8a8.sample(dev, ud)[0])
    assert torch.equal(w8a8.sample(dev, off)[0], w8a8.sample(dev, torch.zeros_like(ud))[0])
    assert torch.equal(w8a8.sample(dev, ud, off)[0], w8a8.sample(dev, ud, 0.0)[0])
    assert torch.equal(w8a8.sample(dev, ud, None, None, None, None)[0], w8a8.sample(dev, ud)[0])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_rows_of_any_alignment(dt):
    l = peaked(5, 3001, dt, 8)
    for ld in (3001, 3003, 3008, 4000):
        check(l, uniform(5), t=0.8, k=50, p=0.9, m=0.01, ld=ld)
    flat = torch.cat([torch.zeros(1), l[0].float()]).to(dt).to(DEV)[1:]  # not 16-byte aligned
    a = w8a8.sample(flat[None], uniform(1).to(DEV), 0.8, 50, 0.9)[0]
    assert int(a) == serving.draw(l[0].float().numpy(), float(uniform(1)), 0.8, 50, np.float32(0.9))[0]


def test_many_rows_and_a_large_vocabulary():
    check(peaked(300, 3000, torch.bfloat16, 9), uniform(300), t=0.9, k=40, p=0.95)
    check(peaked(1, 1 << 20, torch.bfloat16, 10), uniform(1), t=0.9, p=0.95)
    check(peaked(1, (1 << 20) + 5, torch.float32, 11), uniform(1), t=1.3)


def test_draws_follow_the_probabilities():
    """Evenly spaced u hit each kept token in proportion: within one draw."""
    l = torch.log(torch.tensor([0.5, 0.125, 0.25, 0.0625, 0.0625]))
    n = 4096
    u = (torch.arange(n) + 0.5) / n
    t, _ = w8a8.sample(l.expand(n, 5).contiguous().to(DEV), u.to(DEV))
    count = torch.bincount(t, minlength=5).cpu().double() / n
    assert ((count - torch.tensor([0.5, 0.125, 0.25, 0.0625, 0.0625])).abs() <= 1.0 / n).all()


def test_binding_refusals():
    l = torch.zeros((2, 100), dtype=torch.bfloat16, device=DEV)
    u = torch.zeros(2, device=DEV)
    for bad in (dict(logits=l.t()), dict(logits=l.cpu()), dict(u=u[:1]), dict(u=u.double()), dict(temperature=torch.ones(3, device=DEV)),
                dict(top_k=torch.ones(2, dtype=torch.int64, device=DEV)), dict(out=torch.zeros(2, dtype=torch.int32, device=DEV)),
                dict(min_p=torch.ones(2))):
        a = dict(logits=l, u=u)
        a.update(bad)
        with pytest.raises(ValueError):
            w8a8.sample(**a)
    with pytest.raises(TypeError):
        w8a8.sample(l.half(), u)
    with pytest.raises(w8a8.W8A8Error):
        w8a8.sample(l, u, temperature=math.nan)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_prefixes_that_end_far_below_the_largest_logit(dt):
    """More than a thousand bf16 values apart, across 0, with and without the
    other filters; and temperatures that make all weights alike or all but one 0."""
    g = serving.gen(14)
    l = torch.cat([torch.randn((5, 20000), generator=g) * 1e-3, torch.full((5, 4), 8.0)], 1).to(dt)
    check(l, uniform(5), k=torch.tensor([3, 5, 5000, 11000, 20003], dtype=torch.int32))
    check(l, uniform(5), p=torch.tensor([0.2, 0.4, 0.7, 0.99, 0.999999]))
    check(l, uniform(5), m=torch.tensor([1e-7, 1e-3, 3.3e-4, 3.4e-4, 0.5]))
    check(l, uniform(5), k=15000, p=0.9, m=3.36e-4)
    for t in (1e30, math.inf, 1e-30, 2.0 ** -149):
        check(l, uniform(5), t=t)
        check(l, uniform(5), t=t, k=12000, p=0.5)
    l[:, 7] = math.inf
    check(l, uniform(5), t=math.inf)


def test_workspace_refusal():
    l, u = torch.zeros((2, 100), dtype=torch.bfloat16, device=DEV), torch.zeros(2, device=DEV)
    need = w8a8.sample_workspace_bytes(2, 100, torch.bfloat16)
    assert need > 0
    with pytest.raises(w8a8.W8A8Error) as e:
        w8a8.sample(l, u, ws=torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    assert e.value.status == w8a8.EWORKSPACE


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("centre", [0.5, -0.5, 0.0])
@pytest.mark.parametrize("n", [70, 300, 1001, 3001, 9001, 20001])
def test_many_values_close_together(n, centre, dt):
    """Logits within 0.02 of each other, up to thousands of different ones in a bin,
    at odd row starts (-0 among them): every filter ends among them."""
    g = serving.gen(n)
    l = (centre + 0.02 * (torch.rand((4, n), generator=g) - 0.5)).to(dt)
    l[:, ::50] *= -0.0 if centre == 0.0 else 1.0
    u = uniform(4, n)
    check(l, u, k=torch.tensor([1, n // 7, n // 2, n - 1], dtype=torch.int32), ld=n + 3)
    check(l, u, p=torch.tensor([0.001, 0.3, 0.6, 0.995]))
    check(l, u, m=torch.tensor([0.999, 0.993, 0.985, 0.981]))
    check(l, u, t=0.01, k=n // 2, p=0.7, m=0.3)
