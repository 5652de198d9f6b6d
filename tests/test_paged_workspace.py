"""Where the workspace of a paged attention call comes from: on the host with a recording allocator (which stream a block is asked
from), and on the GPU with work pending on the current stream."""
import contextlib
import ctypes

import pytest
import torch

from paper_2604_24432_b200 import binding as ksa
from paper_2604_24432_b200 import build as ksa_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    ksa_build.build()


def _params(**change):
    good = dict(struct_size=ctypes.sizeof(ksa.ksa_paged_params), batch=1, num_rows=1152, chunk_len=8, summaries_per_chunk=1, window_chunks=128,
                num_q_heads=32, num_kv_heads=8, head_dim=128, softmax_scale=0.1, flags=0, kv_format=ksa.KSA_KV_E4M3, page_rows=64,
                num_pages=7, text_cols=600, summ_cols=70, page_stride=65536, head_stride=8192, row_stride=128)
    return bytes(ksa.ksa_paged_params(**{**good, **change}))


def _need(**change):
    n = ctypes.c_size_t()
    assert ksa.lib().ksa_paged_workspace_bytes(_params(**change), ctypes.byref(n)) == 0
    return n.value


def test_a_call_held_to_mma_sync_wants_none():
    assert _need() > 0 and _need(flags=ksa.KSA_FLAG_PAGED_TCGEN05) == _need() and _need(flags=ksa.KSA_FLAG_PAGED_MMA_SYNC) == 0


def test_strides_do_not_matter_to_its_size():
    assert _need(page_stride=0, head_stride=0, row_stride=0) == _need(page_stride=-8, head_stride=3, row_stride=1) == _need()


class Allocator:
    """torch.empty and the streams, recorded: `asked` is the stream of each request."""

    def __init__(self, monkeypatch, current):
        self.on, self.asked = current, []
        monkeypatch.setattr(ksa, "_current_stream", lambda device: self.on)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: 0)
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        monkeypatch.setattr(torch, "empty", self.empty)

    @contextlib.contextmanager
    def stream(self, s):
        before, self.on = self.on, s
        try:
            yield
        finally:
            self.on = before

    def empty(self, n, **kw):
        self.asked.append(self.on)
        return type("Block", (), {"record_stream": lambda self, s: None})()


def _cache():
    c = object.__new__(ksa.PagedCache)
    c.device = torch.device("cuda", 0)
    return c


@pytest.mark.parametrize("current,stream,want", [(7, None, 7), (7, 7, 7), (7, 9, 9), (0, 9, 9), (7, 0, 0), (0, 0, 0)])
def test_block_is_asked_for_on_the_calls_stream(monkeypatch, current, stream, want):
    mem = Allocator(monkeypatch, current)
    assert _cache()._workspace(_params(), stream) is not None
    assert mem.asked == [want] and mem.on == current


@pytest.mark.parametrize("stream", [None, 9])
def test_no_memory_means_no_workspace(monkeypatch, stream):
    mem = Allocator(monkeypatch, 7)

    def full(n, **kw):
        raise torch.OutOfMemoryError("no room")
    monkeypatch.setattr(torch, "empty", full)
    assert _cache()._workspace(_params(), stream) is None and mem.on == 7


@pytest.mark.gpu
def test_pending_work_on_the_current_stream_keeps_its_memory():
    """The current stream is busy and then fills a block of the workspace's size, which the host has freed by the time a call on another
    stream asks for its own."""
    from tests.test_gpu_paged import Server
    ctx = ksa.Context(0)
    s = Server(ctx, 8, 1, 12, 16, 2, 128, 32, "e4m3", [1500], seed=3)
    spans = [(800, 700)]
    s.fill(spans)
    want = s.attn(spans)
    batch, q = s.batch(spans), s.rows(s.q, spans)
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    p = s.cache._params(batch, 700, (0, 0), (0, 0), (0, 0), (0, 0))
    size = s.cache._workspace(p, None).numel()
    side = torch.cuda.Stream()
    for _ in range(5):
        torch.cuda.synchronize()
        x = torch.empty(size, dtype=torch.uint8, device="cuda:0")
        y = torch.empty_like(x)
        torch.cuda._sleep(20_000_000)
        x.fill_(85)
        y.copy_(x)
        del x
        s.cache.attn(batch, q, out, lse, stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert (y == 85).all() and torch.equal(out, want[0]) and torch.equal(lse, want[1])
        out.zero_(), lse.zero_()
    ctx.close()
