"""Refusals and host functions of the serving operators, without a GPU: every
call fails validation before any HIP call.  Also the plain forms themselves
against small cases worked by hand."""

import ctypes
import math

import numpy as np
import pytest
import torch

import serving
from paper_2608_28003_amd import w8a8

P = ctypes.c_void_p
FAKE, MIS4, MIS2 = P(0x1000), P(0x1004), P(0x1002)


def kv(**over):
    a = dict(n_pages=8, page=16, n_kv=1, head_dim=256, k=FAKE, v=FAKE, sk=FAKE, sv=FAKE)
    a.update(over)
    return w8a8.PagedKvDesc(*[a[k] for k in ("n_pages", "page", "n_kv", "head_dim", "k", "v", "sk", "sv")])


def batch(**over):
    a = dict(n_seqs=2, max_pages=4, table=FAKE, q_start=FAKE, ctx_len=FAKE, max_q=4)
    a.update(over)
    return w8a8.PagedBatchDesc(*[a[k] for k in ("n_seqs", "max_pages", "table", "q_start", "ctx_len", "max_q")])


def rope_desc(**over):
    a = dict(head_dim=256, rot_dim=256, layout=0, freq=FAKE, scale=1.0)
    a.update(over)
    return w8a8.RopeDesc(*[a[k] for k in ("head_dim", "rot_dim", "layout", "freq", "scale")])


def each(fn, ok, bads):
    for i, bad, code in bads:
        args = list(ok)
        args[i] = bad
        assert fn(*args) == code, (i, bad, w8a8.lib().w8a8_last_error())


def test_rope_refusals():
    f = w8a8.lib().w8a8_rope
    ok = (rope_desc(), FAKE, w8a8.BF16, 4, 5, 1536, FAKE, FAKE, 1280, None)
    E, U = w8a8.EINVAL, w8a8.EUNSUPPORTED
    each(f, ok, [(0, None, E), (1, None, E), (1, MIS4, E), (7, None, E), (7, MIS4, E), (6, None, E), (6, MIS2, E),
                 (2, 7, U), (3, 0, E), (3, 1 << 26, U), (4, 0, E), (4, 5000, U), (5, 1272, E), (5, 1284, E), (8, 1279, E),
                 (0, rope_desc(head_dim=250), U), (0, rope_desc(head_dim=2048), U), (0, rope_desc(rot_dim=24), U),
                 (0, rope_desc(rot_dim=0), U), (0, rope_desc(rot_dim=272), U), (0, rope_desc(layout=2), U),
                 (0, rope_desc(freq=None), E), (0, rope_desc(freq=MIS4), E), (0, rope_desc(scale=math.inf), E)])
    # in place with two strides: the same pointer twice
    assert f(rope_desc(), FAKE, w8a8.BF16, 4, 5, 1536, MIS2, FAKE, 1280, None) == E


def bad_caches():
    E, U = w8a8.EINVAL, w8a8.EUNSUPPORTED
    return [(None, E), (kv(k=None), E), (kv(v=MIS4), E), (kv(sk=None), E), (kv(sv=None), E), (kv(sk=MIS4), E),
            (kv(head_dim=64), U), (kv(page=8), U), (kv(page=48), U), (kv(page=1 << 17), U), (kv(n_kv=0), E),
            (kv(n_pages=0), E), (kv(n_pages=1 << 31), U)]


def bad_batches():
    E, U = w8a8.EINVAL, w8a8.EUNSUPPORTED
    return [(None, E), (batch(n_seqs=0), E), (batch(max_pages=0), E), (batch(max_q=0), E), (batch(table=None), E),
            (batch(q_start=MIS2), E), (batch(ctx_len=None), E), (batch(n_seqs=1 << 21), U), (batch(max_pages=1 << 27), U)]


def test_append_and_read_refusals():
    L, E, U = w8a8.lib(), w8a8.EINVAL, w8a8.EUNSUPPORTED
    ok = (FAKE, 4, 1536, 4, rope_desc(), kv(), batch(), P(0x2000), 1024, None)
    each(L.w8a8_kv_append, ok, [(0, None, E), (0, MIS4, E), (1, 0, E), (2, 1528, E), (2, 1537, E), (3, 0, E), (7, None, E),
                                (8, 1016, E), (4, rope_desc(head_dim=128, rot_dim=128), E), (4, rope_desc(layout=5), U),
                                (7, FAKE, E)]
         + [(5, b, c) for b, c in bad_caches()] + [(6, b, c) for b, c in bad_batches()])
    ok = (kv(), batch(), 4, FAKE, FAKE, None)
    each(L.w8a8_kv_read, ok, [(2, 0, E), (3, None, E), (4, MIS4, E)]
         + [(0, b, c) for b, c in bad_caches()] + [(1, b, c) for b, c in bad_batches()])


def test_attention_refusals():
    L, E, U = w8a8.lib(), w8a8.EINVAL, w8a8.EUNSUPPORTED
    ok = (FAKE, 4, 1024, 4, kv(), batch(), 1024, 0.0625, FAKE, 1024, FAKE, 1 << 40, None)
    each(L.w8a8_attn_paged, ok, [(0, None, E), (0, MIS4, E), (1, 0, E), (1, 1 << 26, U), (2, 1000, E), (3, 0, E), (6, 0, E),
                                 (7, math.nan, E), (7, math.inf, E), (8, None, E), (9, 1020, E), (4, kv(n_kv=3), E)]
         + [(4, b, c) for b, c in bad_caches()] + [(5, b, c) for b, c in bad_batches()])


def sample_desc(**over):
    a = dict(temperature=None, temperature_all=1.0, top_k=None, top_k_all=0, top_p=None, top_p_all=1.0, min_p=None, min_p_all=0.0)
    a.update(over)
    return w8a8.SampleDesc(*a.values())


def test_sample_refusals():
    L, E, U = w8a8.lib(), w8a8.EINVAL, w8a8.EUNSUPPORTED
    ok = (sample_desc(), FAKE, w8a8.BF16, 4, 1000, 1000, FAKE, FAKE, FAKE, FAKE, 1 << 40, None)
    each(L.w8a8_sample, ok, [(0, None, E), (1, None, E), (1, P(0x1001), E), (2, 5, U), (3, 0, E), (3, 1 << 21, U), (4, 0, E),
                             (4, (1 << 24) + 1, U), (5, 999, E), (6, None, E), (6, MIS2, E), (7, None, E), (7, MIS4, E),
                             (8, MIS2, E), (0, sample_desc(top_k=MIS2), E), (0, sample_desc(temperature_all=math.nan), E),
                             (0, sample_desc(top_p_all=math.nan), E), (0, sample_desc(min_p_all=math.nan), E)])
    args = list(ok)
    args[1], args[2] = MIS2, w8a8.F32
    assert L.w8a8_sample(*args) == E


def test_frequencies():
    for rot in (2, 16, 64, 256):
        f, s = w8a8.rope_frequencies(rot, 10000.0)
        np.testing.assert_allclose(f, 10000.0 ** (-2.0 * np.arange(rot // 2) / rot), rtol=1e-14)
        assert s == 1.0
    f, s = w8a8.rope_frequencies(128, 1e6, "linear", 8.0)
    np.testing.assert_allclose(f * 8.0, w8a8.rope_frequencies(128, 1e6)[0], rtol=1e-15)
    # the base's scaling slows the slowest pair by the factor and leaves the fastest
    f, s = w8a8.rope_frequencies(128, 1e4, "ntk", 4.0)
    g = w8a8.rope_frequencies(128, 1e4)[0]
    assert f[0] == 1.0 and s == 1.0
    np.testing.assert_allclose(f[-1], g[-1] / 4.0, rtol=1e-13)
    # by pair: fast ones kept, slow ones divided, a falling ramp between, scale 1 + 0.1 ln(factor)
    f, s = w8a8.rope_frequencies(128, 1e4, "yarn", 8.0, 4096)
    ratio = g / f
    turns = 4096 * g / (2 * np.pi)
    np.testing.assert_allclose(ratio[turns > 40], 1.0, rtol=1e-14)
    np.testing.assert_allclose(ratio[turns < 0.8], 8.0, rtol=1e-14)
    assert (np.diff(ratio) >= -1e-12).all() and abs(s - (1 + 0.1 * math.log(8.0))) < 1e-7
    np.testing.assert_allclose(w8a8.rope_frequencies(128, 1e4, "yarn", 1.0, 4096)[0], g, rtol=1e-14)


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=15), dict(theta=1.0), dict(theta=math.inf), dict(scaling="other"),
                                 dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=2.0, rot_dim=2),
                                 dict(scaling="yarn", factor=2.0, original=0), dict(scaling="linear", factor=math.nan)])
def test_frequency_refusals(bad):
    a = dict(rot_dim=64)
    a.update(bad)
    with pytest.raises(ValueError):
        w8a8.rope_frequencies(**a)


def test_plain_forms_by_hand():
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0]]], dtype=torch.float64)
    f = torch.tensor([math.pi / 2, 0.0], dtype=torch.float64)
    got = serving.turned(x, torch.tensor([1]), f, 1.0, 4, "half")
    np.testing.assert_allclose(got[0, 0].numpy(), [-3.0, 2.0, 1.0, 4.0], atol=1e-15)
    got = serving.turned(x, torch.tensor([1]), f, 1.0, 4, "interleaved")
    np.testing.assert_allclose(got[0, 0].numpy(), [-2.0, 1.0, 3.0, 4.0], atol=1e-15)
    l = np.log([0.1, 0.4, 0.3, 0.2])
    assert [serving.draw(l, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.79, 0.81)] == [0, 0, 1, 1, 2, 2, 3]
    assert [serving.draw(l, u, top_k=2)[0] for u in (0.0, 0.56, 0.58)] == [1, 1, 2]
    assert [serving.draw(l, u, top_p=0.69)[0] for u in (0.0, 0.9)] == [1, 2]
    assert serving.draw(l, 0.99, min_p=0.6)[0] == 2 and serving.draw(l, 0.99, min_p=0.8)[0] == 1
    assert serving.draw(l, 0.99, temperature=0.0) == (1, 1.0)
    assert serving.draw([1.0, 1.0, 1.0], 0.6, top_k=2)[0] == 1      # the lowest indexes of equal logits
    assert serving.draw([-math.inf, math.nan], 0.5) == (-1, 0.0)
    c, s = serving.codes_of(np.array([[127.0, -63.5, 0.5, 1.5], [0, 0, 0, 0]], np.float32))
    assert c.tolist() == [[127, -64, 0, 2], [0, 0, 0, 0]] and s.tolist() == [1.0, 0.0]
