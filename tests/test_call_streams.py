"""Buffers that a call makes for itself belong to the stream that its kernels run on: filled before them, and not handed out
again before they have passed."""
import contextlib
import types

import numpy as np
import pytest
import torch

import paper_2608_23834_b200 as M

gpu = pytest.mark.gpu


class Recorder:
    """Stands in for streams, allocations and the library, and notes on which stream each buffer was made."""

    def __init__(self, monkeypatch):
        self.current, self.made, self.calls = "caller", [], []
        monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0, name=self.current))
        for name in ("zeros", "empty"):
            monkeypatch.setattr(torch, name, self.noted(getattr(torch, name)))
        monkeypatch.setattr(M, "lib", lambda: self)
        monkeypatch.setattr(M, "_native", types.SimpleNamespace(chunk_attention=lambda *a: 1, append_rotary=lambda *a: 1))

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s.name
        yield
        self.current = before

    def noted(self, make):
        def f(*a, **kw):
            self.made.append((self.current, make(*a, **kw)))
            return self.made[-1][1]
        return f

    def mkv_chunk_workspace_bytes(self, cfg, batch, pages, n):
        n._obj.value = 4096
        return 0

    def mkv_chunk_attention(self, *a):
        self.calls.append(a[-1].value or 0)
        return 0

    mkv_append_rotary = mkv_chunk_attention


def host_pool():
    p = M.Pool.__new__(M.Pool)
    p.d, p.hkv, p.hq, p.handle, p._ref = 128, 1, 2, None, None
    p.cfg = M.make_config(128, 1, 2, 4, 4, np.ones(128, np.int8))
    p.device = torch.device("cpu")
    p.fp8_arena = torch.zeros(16, dtype=torch.uint8)
    return p


CPU = torch.device("cpu")
i32 = lambda *x: torch.tensor(x, dtype=torch.int32)


@pytest.mark.parametrize("given", ["", "out", "workspace"])
def test_buffers_of_chunk_attention_are_made_on_the_launch_stream(monkeypatch, given):
    pool, q = host_pool(), torch.ones(3, 2, 128, dtype=torch.bfloat16)
    kw = {"out": dict(out=torch.ones_like(q)), "workspace": dict(workspace=torch.ones(4096, dtype=torch.uint8))}.get(given, {})
    table, tags = torch.ones(1, 2, dtype=torch.int32), torch.ones(1, 2, dtype=torch.uint8)
    starts, lens = i32(0, 3), i32(20)
    r = Recorder(monkeypatch)
    side = types.SimpleNamespace(name="side", cuda_stream=77, device=CPU)
    pool.chunk_attention(q, starts, table, tags, lens, 1.0, stream=side, **kw)
    assert r.calls == [77] and len(r.made) == (1 if given else 2) and all(s == "side" for s, _ in r.made) and r.current == "caller"
    pool.chunk_attention(q, starts, table, tags, lens, 1.0, **kw)
    assert r.calls == [77, 0] and all(s == "caller" for s, _ in r.made[len(r.made) // 2:])
    elsewhere = types.SimpleNamespace(name="side", cuda_stream=77, device=torch.device("cuda", 5))
    with pytest.raises(AssertionError):
        pool.chunk_attention(q, starts, table, tags, lens, 1.0, stream=elsewhere, **kw)
    assert len(r.calls) == 2


def test_queries_of_append_rotary_are_made_on_the_launch_stream(monkeypatch):
    pool, q = host_pool(), torch.ones(3, 2, 128, dtype=torch.bfloat16)
    rot, pos = M.Rotary(np.ones(64), device="cpu"), i32(0, 1, 2)
    r = Recorder(monkeypatch)
    side = types.SimpleNamespace(name="side", cuda_stream=77, device=CPU)
    out = pool.append_rotary(q, None, None, None, pos, rot, stream=side)
    assert r.calls == [77] and [s for s, _ in r.made] == ["side"] and r.made[0][1] is out and out.shape == q.shape


@gpu
def test_a_side_stream_ahead_of_the_current_one():
    """The side stream's calls pass while the current stream is held up: neither a fill nor a second owner of the workspace may
    come behind them."""
    from test_gpu_chunk import Cache
    c = Cache(128, 2, 4, [(200, 30), (333, 5)], 2, seed=3)
    pool, dev, q = c.pool(), c.device(), c.q.cuda()
    ref = c.reference()
    rot, pos = M.Rotary(np.zeros(64)), torch.zeros(q.shape[0], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    for _ in range(2):                                               # (kernels loaded, memory at hand: nothing below waits for them)
        lse = torch.empty(q.shape[:2], device="cuda")
        pool.append_rotary(q, None, None, None, pos, rot, stream=side)
        pool.chunk_attention(q, *dev, c.scale, lse=lse, stream=side)
        torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                                   # 0.1 s of the current stream
    out = pool.chunk_attention(q, *dev, c.scale, lse=lse, stream=side)
    turned = pool.append_rotary(q, None, None, None, pos, rot, stream=side)
    side.synchronize()
    waited = torch.cuda.current_stream().query()
    with torch.cuda.stream(side):
        early, early_q = out.clone(), turned.clone()
    torch.cuda.synchronize()
    assert not waited, "the current stream was not held up long enough to tell"
    assert torch.equal(out, early) and torch.equal(early_q, q) and torch.equal(turned, q) and pool.status() == M.OK
    c.check(out, lse, ref)
