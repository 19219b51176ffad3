"""Device-memory plumbing around the three entry points.

`SonicBatch` owns the device tensors of one packed batch (inputs, outputs,
workspaces, the compact cache and the status word) and calls the C ABI
through `sonic`.  torch is used only to allocate memory and to provide the
stream; every step of the path runs in libsonic.so.
"""
from __future__ import annotations

import functools
from typing import Optional, Sequence

import numpy as np
import torch

from . import sonic


def bf16_to_device(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """Upload raw bf16 bit patterns (uint16) as a bfloat16 tensor, unchanged."""
    a = np.ascontiguousarray(bits, dtype=np.uint16)
    return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16).to(device)


def bf16_to_host(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def check(code: int, where: str):
    if code != sonic.OK:
        raise sonic.SonicError(code, where)


class SonicBatch:
    """One packed batch on the device.

    role uint8 [T], turn_id int32 [T], cu_seqlens int32 [B+1], q/k/v bf16 bits.
    """

    def __init__(self, role, turn_id, cu_seqlens, q_bits, k_bits, v_bits, device="cuda"):
        self.device = torch.device(device)
        self.cu_host = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        self.batch = len(self.cu_host) - 1
        self.total_tokens = int(self.cu_host[-1])
        self.lengths = np.diff(self.cu_host)
        self.max_seqlen = int(self.lengths.max()) if self.batch else 0
        self.role = torch.from_numpy(np.ascontiguousarray(role, dtype=np.uint8)).to(self.device)
        self.turn_id = torch.from_numpy(np.ascontiguousarray(turn_id, dtype=np.int32)).to(self.device)
        self.cu = torch.from_numpy(self.cu_host).to(self.device)
        self.k = bf16_to_device(k_bits, self.device)
        self.v = bf16_to_device(v_bits, self.device)
        self.T, self.Hkv, self.d = self.k.shape
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        # a decode-only batch has no prefill queries
        self.q = None if q_bits is None else bf16_to_device(q_bits, self.device)
        self.Hq = 0 if self.q is None else self.q.shape[1]
        self.out = None if self.q is None else torch.empty((self.T, self.Hq, self.d), dtype=torch.float32,
                                                           device=self.device)
        ws = sonic.prefill_workspace_bytes(self.batch, self.total_tokens, max(self.Hq, 1), self.Hkv, self.d)
        self.prefill_ws = torch.empty(max(ws, 256), dtype=torch.uint8, device=self.device)
        self.cache = None
        self.cache_q4 = None

    # ------------------------------------------------------------- step 1
    def prefill(self, stream=None, nexus_scope: int = sonic.NEXUS_ALL, nexus_mass=None, key_weight=None) -> int:
        return sonic.segment_attn_prefill(self.cu, self.role, self.turn_id, self.q, self.k, self.v, self.out,
                                          self.prefill_ws, self.status, nexus_scope=nexus_scope,
                                          nexus_mass=nexus_mass, key_weight=key_weight, stream=stream)

    # ------------------------------------------------------------- step 2
    def alloc_cache(self, capacities: Sequence[int], fill_bits: int = 0xFFFF):
        cap = np.asarray(capacities, dtype=np.int64)
        off = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
        rows = int(cap.sum())
        self.cache = CompactCache(rows, self.Hkv, self.d, off, cap.astype(np.int32), self.device, fill_bits)
        return self.cache

    def compact(self, stream=None) -> int:
        c = self.cache
        return sonic.kv_compact(self.cu, self.role, self.k, self.v, c.k, c.v, c.row_off, c.row_cap, c.length,
                                c.keep_idx, self.status, self.max_seqlen, stream=stream)

    def alloc_cache_q4(self, capacities: Sequence[int]):
        cap = np.asarray(capacities, dtype=np.int64)
        off = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
        self.cache_q4 = Q4Cache(int(cap.sum()), self.Hkv, self.d, off, cap.astype(np.int32), self.device)
        return self.cache_q4

    def compact_q4(self, stream=None) -> int:
        c = self.cache_q4
        return sonic.kv_compact_q4(self.cu, self.role, self.k, self.v, c.k, c.k_scale, c.v, c.v_scale, c.row_off, c.row_cap,
                                   c.length, c.keep_idx, self.status, self.max_seqlen, stream=stream)

    def read_status(self) -> int:
        return int(self.status.item())

    def clear_status(self):
        self.status.zero_()


class _Workspaces:
    """Device workspaces of a cache's calls.

    One is made on the stream of the call that first needs it, so that its zeros are in place for that call, and kept
    as long as the cache: a larger one does not replace it for what is still running on a stream or was captured into a
    graph.  Sizes double, so the smaller ones add up to no more than the last.
    """

    def __init__(self):
        self.made = {}

    def get(self, key, nbytes: int, device, stream, counters: int = 0) -> torch.Tensor:
        """A workspace of nbytes or more for calls of one key (the numbers that its counters' places depend on);
        `counters`: its bytes from the start on that have to be zero before the first call, which leaves them so."""
        fits = [w for w in self.made.get(key, ()) if w.numel() >= nbytes]
        if fits:
            return fits[-1]
        with torch.cuda.stream(stream):
            # zeros written under capture are there only when that graph runs: such a workspace is for captured calls,
            # each of which clears the counters itself
            if counters and torch.device(device).type == "cuda" and torch.cuda.is_current_stream_capturing():
                ws = self.get((key, "captured"), nbytes, device, stream)
            else:
                mine = self.made.setdefault(key, [])
                mine.append(torch.empty(max(nbytes, 256, 2 * mine[-1].numel() if mine else 0), dtype=torch.uint8, device=device))
                ws = mine[-1]
            ws[:counters].zero_()
        return ws


@functools.lru_cache(maxsize=1024)
def _bytes(size, *shape) -> int:
    return size(*shape)


def _counter_bytes(batch: int, num_kv_heads: int) -> int:
    """The completion counters' share of a decode workspace: int32 per request and per (request, kv-head), each array on
    256 bytes."""
    return sum((4 * n + 255) // 256 * 256 for n in (batch, batch * num_kv_heads))


def _places(rows, row_off, row_cap, device):
    """Of every cache row, on the device: the first row of the request that owns it (int64), and its place in it (int32)."""
    first, place = np.zeros(rows, np.int64), np.arange(rows, dtype=np.int32)
    for o, n in zip(row_off, row_cap):
        place[o:o + n] -= place[o:o + 1]
        first[o:o + n] = o
    return torch.from_numpy(first).to(device), torch.from_numpy(place).to(device)


def _evict(cache, keep_head, keep_tail, budget, status, stream, **scales) -> int:
    """sonic.cache_evict in place; keep_idx moves with the rows, so that each still names its prompt position."""
    n = int(cache.row_cap_host.max()) if cache.batch else 0
    ws = cache.workspaces.get("evict", sonic.cache_evict_workspace_bytes(cache.batch, n), cache.k.device, stream)
    with torch.cuda.stream(stream):
        moved = cache.place.clone()   # where nothing moves: each row's own
        st = sonic.cache_evict(cache.k, cache.v, cache.row_off, cache.length, cache.row_weight, keep_head, keep_tail, budget, ws,
                               status, n, keep_idx=moved, stream=stream, **scales)
        if st == sonic.OK:
            cache.keep_idx.copy_(cache.keep_idx[(cache.first_row + moved).clamp_(max=moved.numel() - 1)])
    return st


def _tree_decode(cache, plan, q, k_new, v_new, out, status, max_nodes, max_ctx, stream, **scales) -> int:
    n = _bytes(sonic.tree_decode_workspace_bytes, cache.batch, int(max_nodes), q.shape[1], q.shape[2], int(max_ctx))
    ws = cache.workspaces.get("tree", n, q.device, stream)
    return sonic.tree_decode(plan, cache.k, cache.v, cache.row_off, cache.length, q, k_new, v_new, out, ws, status, max_nodes, max_ctx,
                             stream=stream, **scales)


class CompactCache:
    """Per-request cache rows [row_off[b], row_off[b] + row_cap[b]) of a [rows, Hkv, d] bf16 pair.

    row_weight (fp32 [rows], for decode_weighted and evict; None until decode_weighted or the caller makes it) is the caller's
    to set after a compaction: sonic.kv_compact_weights, or zeros."""

    def __init__(self, rows, Hkv, d, row_off, row_cap, device, fill_bits=0xFFFF):
        self.rows, self.Hkv, self.d = rows, Hkv, d
        fill = np.int16(np.uint16(fill_bits).view(np.int16))
        self.k = torch.full((max(rows, 1), Hkv, d), int(fill), dtype=torch.int16, device=device).view(torch.bfloat16)
        self.v = torch.full((max(rows, 1), Hkv, d), int(fill), dtype=torch.int16, device=device).view(torch.bfloat16)
        self.keep_idx = torch.full((max(rows, 1),), -1, dtype=torch.int32, device=device)
        self.row_off_host = np.asarray(row_off, dtype=np.int64)
        self.row_cap_host = np.asarray(row_cap, dtype=np.int32)
        self.row_off = torch.from_numpy(self.row_off_host).to(device)
        self.row_cap = torch.from_numpy(self.row_cap_host).to(device)
        self.length = torch.zeros(len(row_cap), dtype=torch.int32, device=device)
        self.batch = len(row_cap)
        self.first_row, self.place = _places(self.keep_idx.numel(), self.row_off_host, self.row_cap_host, device)
        self.workspaces = _Workspaces()
        self.row_weight = None

    def decode(self, q, k_new, v_new, out, status, max_ctx: int, row_role: Optional[torch.Tensor] = None,
               stream=None) -> int:
        ws = self._decode_ws(_bytes(sonic.decode_workspace_bytes, *q.shape, int(max_ctx)), k_new, stream)
        return sonic.compressed_decode(self.k, self.v, self.row_off, self.row_cap, self.length, q, k_new, v_new,
                                       out, ws, status, max_ctx, row_role=row_role, stream=stream)

    def _decode_ws(self, nbytes, k_new, stream):
        B, Hkv = k_new.shape[:2]
        return self.workspaces.get(("decode", B, Hkv), nbytes, k_new.device, stream, _counter_bytes(B, Hkv))

    def decode_weighted(self, q, k_new, v_new, out, status, max_ctx: int, stream=None) -> int:
        """decode that also adds each row's attention to row_weight."""
        if self.row_weight is None:
            with torch.cuda.stream(stream):
                if q.is_cuda and torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("set row_weight before capturing: zeros made here would be written again by every replay")
                self.row_weight = torch.zeros(self.k.shape[0], dtype=torch.float32, device=q.device)
        ws = self._decode_ws(_bytes(sonic.decode_weighted_workspace_bytes, *q.shape, int(max_ctx)), k_new, stream)
        return sonic.compressed_decode_weighted(self.k, self.v, self.row_off, self.row_cap, self.length, q, k_new, v_new, out,
                                                self.row_weight, ws, status, max_ctx, stream=stream)

    def tree_decode(self, plan, q, k_new, v_new, out, status, max_nodes: int, max_ctx: int, stream=None) -> int:
        """The attention of drafted tokens over the cache and their own paths; the cache stays as it is.  A cache's calls share
        a workspace: side by side (on two streams, in two graphs) take sonic.tree_decode with one each."""
        return _tree_decode(self, plan, q, k_new, v_new, out, status, max_nodes, max_ctx, stream)

    def append(self, new_cu, k_new, v_new, status, max_rows: int, select=None, select_len=None, stream=None) -> int:
        """New rows to the end of the cache: all of a request's, or those at select.  row_weight and keep_idx of the rows are
        the caller's to set before the next evict or decode_weighted: they hold what a dropped row left there.  With `old` the
        lengths before and `request` each row's request, the new rows are (place >= old[request]) & (place < length[request])."""
        return sonic.cache_append(new_cu, k_new, v_new, self.k, self.v, self.row_off, self.row_cap, self.length, status, max_rows,
                                  select=select, select_len=select_len, stream=stream)

    def evict(self, keep_head, keep_tail, budget, status, stream=None) -> int:
        """Drop the rows of least row_weight, in place; keep_head, keep_tail, budget: int32 [B] on the device.  keep_idx
        goes with the rows."""
        return _evict(self, keep_head, keep_tail, budget, status, stream)


class Q4Cache:
    """The same rows in 4 bits: codes [rows, Hkv, d / 2] and scale bytes [rows, Hkv, d / 32] of K and V.  row_weight as in
    CompactCache, zeros at first."""

    def __init__(self, rows, Hkv, d, row_off, row_cap, device):
        self.rows, self.Hkv, self.d = rows, Hkv, d
        n = max(rows, 1)

        def plane(width):
            return torch.full((n, Hkv, width), 255, dtype=torch.uint8, device=device)   # NaN until written

        self.k, self.k_scale, self.v, self.v_scale = plane(d // 2), plane(d // 32), plane(d // 2), plane(d // 32)
        self.keep_idx = torch.full((n,), -1, dtype=torch.int32, device=device)
        self.row_weight = torch.zeros(n, dtype=torch.float32, device=device)
        self.row_off_host = np.asarray(row_off, dtype=np.int64)
        self.row_cap_host = np.asarray(row_cap, dtype=np.int32)
        self.row_off = torch.from_numpy(self.row_off_host).to(device)
        self.row_cap = torch.from_numpy(self.row_cap_host).to(device)
        self.length = torch.zeros(len(row_cap), dtype=torch.int32, device=device)
        self.batch = len(row_cap)
        self.first_row, self.place = _places(self.keep_idx.numel(), self.row_off_host, self.row_cap_host, device)
        self.workspaces = _Workspaces()

    def decode(self, q, k_new, v_new, out, status, max_ctx: int, weighted: bool = False, stream=None) -> int:
        B, Hkv = k_new.shape[:2]
        n = _bytes(sonic.decode_q4_workspace_bytes, *q.shape, int(max_ctx), weighted)
        ws = self.workspaces.get(("decode", B, Hkv), n, q.device, stream, _counter_bytes(B, Hkv))
        return sonic.compressed_decode_q4(self.k, self.k_scale, self.v, self.v_scale, self.row_off, self.row_cap, self.length, q,
                                          k_new, v_new, out, ws, status, max_ctx,
                                          row_weight=self.row_weight if weighted else None, stream=stream)

    def expand(self, row_begin, row_end, k, v, out_row_off, out_row_cap, status, max_rows: int, stream=None) -> int:
        return sonic.cache_expand_q4(self.k, self.k_scale, self.v, self.v_scale, self.row_off, self.row_cap, row_begin, row_end, k,
                                     v, out_row_off, out_row_cap, status, max_rows, stream=stream)

    def tree_decode(self, plan, q, k_new, v_new, out, status, max_nodes: int, max_ctx: int, stream=None) -> int:
        """The attention of drafted tokens over the cache and their own paths, at the 4-bit values of their rows; the cache
        stays as it is, and its calls share a workspace, as CompactCache's."""
        return _tree_decode(self, plan, q, k_new, v_new, out, status, max_nodes, max_ctx, stream, k_scale=self.k_scale,
                            v_scale=self.v_scale)

    def append(self, new_cu, k_new, v_new, status, max_rows: int, select=None, select_len=None, stream=None) -> int:
        """New rows, rounded, to the end of the cache: all of a request's, or those at select.  row_weight and keep_idx of the
        rows are the caller's to set, as in CompactCache.append."""
        return sonic.cache_append(new_cu, k_new, v_new, self.k, self.v, self.row_off, self.row_cap, self.length, status, max_rows,
                                  select=select, select_len=select_len, k_scale=self.k_scale, v_scale=self.v_scale, stream=stream)

    def evict(self, keep_head, keep_tail, budget, status, stream=None) -> int:
        """Drop the rows of least row_weight, in place; keep_head, keep_tail, budget: int32 [B] on the device.  keep_idx
        goes with the rows."""
        return _evict(self, keep_head, keep_tail, budget, status, stream, k_scale=self.k_scale, v_scale=self.v_scale)


class DraftStep:
    """A step over drafted tokens of `batch` requests, up to total_nodes of them and max_nodes a request: what is made once
    and used by every layer and every step (the plan, the confirmed paths, the logits' workspace): one step at a time.

    plan_trees, then CompactCache.tree_decode (or Q4Cache's) per layer with `plan`, `logits`, `accept`, and the caches'
    append with path and path_len."""

    def __init__(self, batch: int, total_nodes: int, max_nodes: int, device="cuda"):
        self.batch, self.total_nodes, self.max_nodes = batch, total_nodes, max_nodes

        def ints(n):
            return torch.zeros(n, dtype=torch.int32, device=device)

        self.plan = torch.zeros(sonic.tree_plan_bytes(batch, total_nodes, max_nodes), dtype=torch.uint8, device=device)
        self.path, self.path_len, self.next_token = ints(total_nodes), ints(batch), ints(batch)
        self.best = ints(total_nodes)
        self.workspaces = _Workspaces()

    def plan_trees(self, cu_nodes, parent, status, stream=None) -> int:
        return sonic.tree_plan(cu_nodes, parent, self.total_nodes, self.max_nodes, self.plan, status, stream=stream)

    def logits(self, logits, status, stream=None, **how) -> int:
        """sonic.logits_process on the nodes' logits [total_nodes, V]: their best tokens to `best`."""
        n = _bytes(sonic.logits_process_workspace_bytes, *logits.shape)
        ws = self.workspaces.get("logits", n, logits.device, stream)
        return sonic.logits_process(logits, self.best, ws, status, plan=self.plan, batch=self.batch, max_nodes=self.max_nodes,
                                    stream=stream, **how)

    def accept(self, parent, node_token, status, chosen=None, stream=None, **history) -> int:
        """The nodes that `chosen` (by default the best tokens) confirms, to path, path_len and next_token."""
        return sonic.tree_accept(self.plan, parent, node_token, self.best if chosen is None else chosen, self.path, self.path_len,
                                 self.next_token, status, self.max_nodes, stream=stream, **history)
