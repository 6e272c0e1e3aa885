"""Calls with tensors on another device than the current one (no GPU: the library is stood in for)."""

import contextlib
import gc
import weakref

import pytest
import torch

from paper_2605_01910_amd import santa as S


def test_the_workspace_is_cleared_on_its_own_device(monkeypatch):
    """alloc_attend_workspace on device 1 while device 0 is current: the clearing kernel runs on
    device 1's stream with device 1 current."""
    current, calls = [0], []

    class Library:
        def santa_attend_workspace_size(self, *args):
            return 1024

        def santa_workspace_init(self, ws, n, stream):
            calls.append((current[0], n, getattr(stream, "value", stream)))
            return 0

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    empty = torch.empty
    monkeypatch.setattr(S, "load", Library)
    monkeypatch.setattr(S, "_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 1)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: 100 + current[0])
    ws = S.alloc_attend_workspace(None, None, device="cuda:1")
    assert calls == [(1, 1024, 101)] and current == [0]
    assert ws.numel() == 1024 and ws.data_ptr() % 256 == 0


def test_a_chunk_keeps_its_tensor(monkeypatch):
    """chunk_of over a temporary: the prefix sums live as long as the chunk, and a call refuses them on
    another device than its rows."""
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    ends = torch.tensor([0, 5], dtype=torch.int32)
    gone = weakref.ref(ends)
    chunk = S.chunk_of(ends, 5)
    del ends
    gc.collect()
    assert gone() is not None and chunk.q_start == gone().data_ptr()
    rows = torch.zeros(5, 1, 128)
    monkeypatch.setattr(S, "load", lambda: type("L", (), {"santa_attend_chunk": None, "santa_rope_append": None})())
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 1 if self is gone() else 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    shape, kv = S.santa_shape_t(1, 1, 1, 128, S.SANTA_F32), S.santa_kv_t()
    with pytest.raises(ValueError, match="one device"):
        S.santa_attend_chunk(rows, kv, shape, chunk, None, 0.1, rows, rows)
    with pytest.raises(ValueError, match="one device"):
        S.santa_rope_append(rows, rows, rows, kv, shape, chunk, None, rows)
    del chunk
    gc.collect()
    assert gone() is None
