"""Refusals of the serving operators' binding, without a GPU: tensors that claim to
be on one, and a library that only records what it is called with."""

import pytest
import torch

from paper_2608_28003_amd import w8a8


class OnGpu(torch.Tensor):
    """A CPU tensor that the binding takes for one on a GPU."""

    is_cuda = property(lambda self: True)


class Recorder:
    """Stands for the library: every launch is a call in `calls`."""

    def __init__(self):
        self.calls = []

    def w8a8_sample_workspace_bytes(self, *a):
        return 256

    def w8a8_sample(self, *a):
        self.calls.append(a)
        return 0

    w8a8_attn_paged_workspace_bytes = w8a8_sample_workspace_bytes
    w8a8_attn_paged = w8a8_sample


class Stream:
    def __init__(self, *a):
        pass

    def __enter__(self):
        return 0

    def __exit__(self, *a):
        pass


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(w8a8, "lib", lambda: r)
    monkeypatch.setattr(w8a8, "_on", Stream)
    return r


def gpu(t):
    return t.as_subclass(OnGpu)


def test_sample_refuses_rows_that_overlap(recorder):
    """Rows closer together than a row is long: one row expanded, windows over a
    vector.  A call with n for their stride would read behind the tensor."""
    for dt in (torch.bfloat16, torch.float32):
        one = torch.zeros(3000, dtype=dt)
        for l in (one.expand(64, 3000), one.as_strided((64, 1000), (8, 1)), one.as_strided((3, 1000), (999, 1)),
                  one[:1].expand(64, 1)):
            with pytest.raises(ValueError):
                w8a8.sample(gpu(l), torch.zeros(l.shape[0]))
    assert recorder.calls == []


def test_sample_passes_the_stride_there_is(recorder):
    flat = torch.zeros(6000, dtype=torch.bfloat16)
    for l, ld in ((flat.view(6, 1000), 1000), (flat.view(6, 1000)[:, :900], 1000), (flat.view(6, 1000)[::2], 2000),
                  (flat[:1000].expand(1, 1000), 1000), (flat.as_strided((1, 7), (3, 1)), 7), (flat.view(6, 1000)[:, :1], 1000)):
        w8a8.sample(gpu(l), torch.zeros(l.shape[0]))
        a = recorder.calls.pop()
        assert a[1:6] == (l.data_ptr(), w8a8.BF16, *l.shape, ld)


def test_attention_refuses_a_scale_that_overflows():
    """The kernels take scale * log2(e)."""
    from test_serving_host import FAKE, batch, kv

    for scale in (3e38, -2.4e38):
        assert w8a8.lib().w8a8_attn_paged(FAKE, 4, 1024, 4, kv(), batch(), 1024, scale, FAKE, 1024, FAKE, 1 << 40,
                                          None) == w8a8.EINVAL


def test_workspaces_are_memory_of_their_size(recorder):
    """One byte expanded, or every second byte, has as many elements as a workspace of
    that size, but not its memory."""
    logits, u = gpu(torch.zeros(2, 100, dtype=torch.bfloat16)), torch.zeros(2)
    q = gpu(torch.zeros(2, 4, 256, dtype=torch.bfloat16))
    cache = w8a8.PagedKV.empty(2, 16, device="cpu")
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)
    batch = w8a8.PagedBatch(ints([0, 1]), ints(0, 2), ints(20), 2)
    one = torch.zeros(1, dtype=torch.uint8)
    for ws in (one.expand(1 << 20), torch.zeros(1 << 10, dtype=torch.uint8)[::2], torch.zeros(64, 64).t()[1:]):
        with pytest.raises(ValueError):
            w8a8.sample(logits, u, ws=ws)
        with pytest.raises(ValueError):
            w8a8.attn_paged(q, cache, batch, out=q, ws=ws)
    assert recorder.calls == []
    ws = torch.zeros(1 << 10, dtype=torch.int32)
    w8a8.sample(logits, u, ws=ws)
    w8a8.attn_paged(q, cache, batch, out=q, ws=ws)
    assert [a[-3:-1] for a in recorder.calls] == [(ws.data_ptr(), 4 << 10)] * 2
