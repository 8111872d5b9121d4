"""Memory that the binding allocates for a call on a given stream: taken on that stream, and kept
from its next user until the caller's stream is done with it (stand-ins for CUDA's, no GPU)."""
import contextlib

import pytest
import torch

from paper_2607_06601_gb300 import trr


class Streams:
    """Which stream is current, and what was allocated and recorded where."""

    def __init__(self, monkeypatch):
        self.now, self.made, self.recorded = "caller", [], []
        empty = torch.empty

        @contextlib.contextmanager
        def stream(s):
            before, self.now = self.now, s
            yield
            self.now = before

        def made(*args, **kw):
            t = empty(*args, **kw)
            self.made.append((t.data_ptr(), self.now))
            return t

        monkeypatch.setattr(torch.cuda, "stream", stream)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.now)
        monkeypatch.setattr(torch, "empty", made)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.recorded.append((t.data_ptr(), s)))


@pytest.fixture
def cache(monkeypatch):
    c = object.__new__(trr.Cache)
    c.handle, c.pool, c.Hq, c.d, c.head_modes, c._workspace = None, torch.zeros(1), 4, 64, 0, None
    monkeypatch.setattr(trr, "trr_workspace_bytes", lambda handle: 512)
    for name in ("decode_attn", "decode_step", "decode_attn_routed", "decode_attn_sinks", "decode_attn_shared", "fork", "compact"):
        monkeypatch.setattr(trr, "trr_" + name, lambda *a: None)
    return c


N = torch.zeros(3, dtype=torch.int32)
Q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
CALLS = dict(decode_attn=lambda c, s: c.decode_attn(0, N, N, Q, N, stream=s), decode_step=lambda c, s: c.decode_step(0, N, N, Q, Q, N, N, Q, stream=s),
             decode_attn_routed=lambda c, s: c.decode_attn_routed(0, N, N, Q, N, stream=s),
             decode_attn_sinks=lambda c, s: c.decode_attn_sinks(0, N, N, Q, N, 2, stream=s),
             decode_attn_shared=lambda c, s: c.decode_attn_shared(0, N, N, Q, N, N, stream=s))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_rows_and_workspace_belong_to_the_stream_of_the_call(monkeypatch, cache, name):
    streams = Streams(monkeypatch)
    out = CALLS[name](cache, "other")
    here = [(out.data_ptr(), "other")]
    if name in ("decode_attn_sinks", "decode_attn_shared"):
        here.append((cache.workspace().data_ptr(), "other"))
    assert sorted(streams.made) == sorted(here)
    assert sorted(streams.recorded) == sorted((p, "caller") for p, _ in here)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_on_the_current_stream_nothing_is_recorded(monkeypatch, cache, name):
    streams = Streams(monkeypatch)
    CALLS[name](cache, None)
    CALLS[name](cache, "caller")
    assert streams.made and all(s == "caller" for _, s in streams.made) and not streams.recorded


@pytest.mark.parametrize("call", [lambda c, s: c.fork(N, N, N, stream=s), lambda c, s: c.compact(stream=s)])
def test_page_operations_allocate_their_workspace_once_on_their_stream(monkeypatch, cache, call):
    streams = Streams(monkeypatch)
    call(cache, "other")
    call(cache, None)
    assert streams.made == [(cache.workspace().data_ptr(), "other")]
