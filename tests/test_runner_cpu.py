"""The workspaces of the cache classes: made on the stream of the call, and kept while anything may still use them.
The entry points are replaced by a recorder, so this runs without a GPU."""
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2601_21927_amd import runner, sonic
from paper_2601_21927_amd.runner import CompactCache, Q4Cache

B, HQ, HKV, D = 3, 8, 2, 64


class Recorder:
    """Stands in for the stream context and the entry points."""

    def __init__(self, monkeypatch):
        self.active, self.allocated, self.used = None, [], []
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        for name in ("zeros", "empty"):
            monkeypatch.setattr(runner.torch, name, self.allocating(getattr(torch, name)))
        for name in ("compressed_decode", "compressed_decode_weighted", "compressed_decode_q4", "cache_evict"):
            monkeypatch.setattr(sonic, name, self.entry)

    def stream(self, s):
        rec = self

        class Active:
            def __enter__(self):
                self.before, rec.active = rec.active, s or rec.active

            def __exit__(self, *_):
                rec.active = self.before

        return Active()

    def allocating(self, fn):
        def make(*a, **kw):
            self.allocated.append(self.active)
            return fn(*a, **kw)
        return make

    def entry(self, *args, **kw):
        ws = next(a for a in args if torch.is_tensor(a) and a.dtype == torch.uint8 and a.dim() == 1)
        self.used.append((weakref.ref(ws), ws.data_ptr(), ws.numel()))
        return sonic.OK


def caches():
    cap = np.array([900, 20, 300])
    off = np.array([0, 900, 920])
    return [CompactCache(1220, HKV, D, off, cap, "cpu"), Q4Cache(1220, HKV, D, off, cap, "cpu")]


def calls(c):
    """name -> call(max_ctx, stream) of a cache."""
    q, k, out = (torch.full((B, h, D), 0.5, dtype=t) for h, t in ((HQ, torch.bfloat16), (HKV, torch.bfloat16), (HQ, torch.float32)))
    n = torch.ones(B, dtype=torch.int32)
    status = torch.ones(1, dtype=torch.int32)
    new = dict(evict=lambda m, s: c.evict(n, n, n, status, stream=s), decode=lambda m, s: c.decode(q, k, k, out, status, m, stream=s))
    if isinstance(c, Q4Cache):
        new["weighted"] = lambda m, s: c.decode(q, k, k, out, status, m, weighted=True, stream=s)
    else:
        new["weighted"] = lambda m, s: c.decode_weighted(q, k, k, out, status, m, stream=s)
    return new


@pytest.mark.parametrize("name", ["evict", "decode", "weighted"])
@pytest.mark.parametrize("kind", [0, 1])
def test_what_a_call_allocates_is_made_on_its_stream(kind, name, monkeypatch):
    call = calls(caches()[kind])[name]
    rec = Recorder(monkeypatch)
    side = object()
    assert call(900, side) == sonic.OK
    assert rec.allocated and all(s is side for s in rec.allocated)


@pytest.mark.parametrize("name", ["evict", "decode", "weighted"])
@pytest.mark.parametrize("kind", [0, 1])
def test_workspaces_outlive_the_calls_that_use_them(kind, name, monkeypatch):
    cache = caches()[kind]
    call = calls(cache)[name]
    rec = Recorder(monkeypatch)
    for bound in (900, 90000, 900, 2000000):
        assert call(bound, None) == sonic.OK
    gc.collect()
    assert all(ref() is not None for ref, _, _ in rec.used)


@pytest.mark.parametrize("kind", [0, 1])
def test_calls_of_one_shape_share_a_workspace(kind, monkeypatch):
    cache = caches()[kind]
    c = calls(cache)
    rec = Recorder(monkeypatch)
    for name in ("weighted", "decode", "weighted", "decode"):
        assert c[name](900, None) == sonic.OK
    assert len({p for _, p, _ in rec.used}) == 1


@pytest.mark.parametrize("kind", [0, 1])
def test_growing_bounds_take_no_more_than_twice_the_last_workspace(kind, monkeypatch):
    cache = caches()[kind]
    c = calls(cache)
    rec = Recorder(monkeypatch)
    for bound in range(300, 60000, 700):
        assert c["weighted"](bound, None) == sonic.OK
    sizes = {p: n for _, p, n in rec.used}
    need = sonic.decode_q4_workspace_bytes(B, HQ, D, 59999, True) if kind else sonic.decode_weighted_workspace_bytes(B, HQ, D, 59999)
    assert sum(sizes.values()) <= 4 * need


def test_counters_start_at_zero():
    w = runner._Workspaces()
    first = w.get("a", 4096, "cpu", None, 512)
    assert not first[:512].any()
    first.fill_(7)
    assert w.get("a", 4000, "cpu", None, 512) is first and w.get("b", 4000, "cpu", None, 512) is not first
    larger = w.get("a", 5000, "cpu", None, 512)
    assert larger.numel() >= 8192 and not larger[:512].any() and w.get("a", 10, "cpu", None, 512) is larger
