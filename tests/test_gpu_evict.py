"""Eviction by attention weight on the GPU: kept rows, their order, bytes and weights, exactly as the oracle's."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import compaction as OC
from oracle import evict as OE
from oracle import extend as OX
from oracle import q4 as OQ
from oracle.attention import bf16_bits_to_f64
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import CompactCache, Q4Cache, bf16_to_device, bf16_to_host
from tests import gpu_helpers as H

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Rows:
    """A cache of random bytes, on the device and on the host."""

    def __init__(self, rng, lens, extra, Hkv, d, q4, weight=None):
        self.lens, self.q4 = np.asarray(lens), q4
        self.cap = self.lens + extra
        self.off = np.concatenate([[0], np.cumsum(self.cap)[:-1]]).astype(np.int64)
        n = max(int(self.cap.sum()), 1)
        if q4:
            shapes = dict(k=(n, Hkv, d // 2), ks=(n, Hkv, d // 32), v=(n, Hkv, d // 2), vs=(n, Hkv, d // 32))
            self.host = {name: rng.integers(0, 255, size=s).astype(np.uint8) for name, s in shapes.items()}
            self.dev = {name: torch.from_numpy(x.copy()).cuda() for name, x in self.host.items()}
        else:
            self.host = {name: rng.integers(0, 65536, size=(n, Hkv, d)).astype(np.uint16) for name in ("k", "v")}
            self.dev = {name: bf16_to_device(x.copy()) for name, x in self.host.items()}
        self.weight = (rng.random(n) ** 4).astype(np.float32) if weight is None else np.resize(np.asarray(weight, np.float32), n)
        self.row_weight = torch.from_numpy(self.weight.copy()).cuda()
        self.row_off = torch.from_numpy(self.off).cuda()
        self.length = i32(self.lens)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.max_rows = max(int(self.cap.max()), 0)
        # garbage in the workspace: its contents need no initialisation
        self.ws = torch.full((sonic.cache_evict_workspace_bytes(len(lens), self.max_rows),), 0x5A, dtype=torch.uint8, device="cuda")

    def bytes(self, name):
        t = self.dev[name]
        return t.cpu().numpy() if self.q4 else bf16_to_host(t)

    def args(self, head, tail, budget):
        B = len(self.lens)
        hv, tv, bv = (i32(np.broadcast_to(x, B)) for x in (head, tail, budget))
        return (self.dev["k"], self.dev["v"], self.row_off, self.length, self.row_weight, hv, tv, bv, self.ws, self.status,
                self.max_rows), dict(k_scale=self.dev.get("ks"), v_scale=self.dev.get("vs"))

    def kept(self, head, tail, budget):
        B = len(self.lens)
        h, t, b = (np.broadcast_to(x, B) for x in (head, tail, budget))
        return [OE.kept_rows(self.weight[o:o + n], int(h[i]), int(t[i]), int(b[i])) for i, (o, n) in enumerate(zip(self.off, self.lens))]


def check_in_place(r, head, tail, budget):
    a, kw = r.args(head, tail, budget)
    idx = torch.full((r.row_weight.numel(),), -1, dtype=torch.int32, device="cuda")
    assert sonic.cache_evict(*a, **kw, keep_idx=idx) == sonic.OK
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    kept = r.kept(head, tail, budget)
    assert np.array_equal(r.length.cpu().numpy(), [len(x) for x in kept])
    want_w, want_i = r.weight.copy(), np.full(len(r.weight), -1, np.int32)
    for o, rows in zip(r.off, kept):
        want_w[o:o + len(rows)] = r.weight[o + rows]
        want_i[o:o + len(rows)] = rows
    assert np.array_equal(idx.cpu().numpy(), want_i)
    assert np.array_equal(r.row_weight.cpu().numpy(), want_w, equal_nan=True)
    for name, x in r.host.items():
        want = x.copy()
        for o, rows in zip(r.off, kept):
            want[o:o + len(rows)] = x[o + rows]
        assert np.array_equal(r.bytes(name), want), name     # rows behind the kept ones hold what they held


def away_cache(r, caps):
    n = max(int(np.sum(caps)), 1)
    out = {name: torch.zeros((n,) + x.shape[1:], dtype=x.dtype, device="cuda") for name, x in r.dev.items()}
    off = np.concatenate([[0], np.cumsum(caps)[:-1]]).astype(np.int64)
    more = dict(k_out=out["k"], v_out=out["v"], k_scale_out=out.get("ks"), v_scale_out=out.get("vs"), out_row_off=torch.from_numpy(off).cuda(),
                out_row_cap=i32(caps), out_len=i32([-5] * len(caps)), out_weight=torch.full((n,), -3.0, device="cuda"),
                keep_idx=torch.full((n,), -1, dtype=torch.int32, device="cuda"))
    return out, off, more


def check_away(r, head, tail, budget):
    kept = r.kept(head, tail, budget)
    caps = np.array([len(x) for x in kept]) + np.arange(len(kept)) % 3
    out, off, more = away_cache(r, caps)
    a, kw = r.args(head, tail, budget)
    assert sonic.cache_evict(*a, **kw, **more) == sonic.OK
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    assert np.array_equal(more["out_len"].cpu().numpy(), [len(x) for x in kept])
    want_i, want_w = np.full(more["keep_idx"].numel(), -1), np.full(more["keep_idx"].numel(), -3.0, np.float32)
    for o, src, rows in zip(off, r.off, kept):
        want_i[o:o + len(rows)], want_w[o:o + len(rows)] = rows, r.weight[src + rows]
    assert np.array_equal(more["keep_idx"].cpu().numpy(), want_i)
    assert np.array_equal(more["out_weight"].cpu().numpy(), want_w, equal_nan=True)
    for name, x in r.host.items():
        got = out[name].cpu().numpy() if r.q4 else bf16_to_host(out[name])
        want = np.zeros_like(got)
        for o, src, rows in zip(off, r.off, kept):
            want[o:o + len(rows)] = x[src + rows]
        assert np.array_equal(got, want), name
        assert np.array_equal(r.bytes(name), x)              # the first cache is left as it is
    assert np.array_equal(r.length.cpu().numpy(), r.lens)


@pytest.mark.parametrize("check", [check_in_place, check_away])
@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("Hkv,d", [(8, 128), (1, 64), (5, 64), (3, 128), (2, 64)])
def test_lengths_and_budgets(Hkv, d, q4, check):
    H.need_gpu()
    rng = np.random.default_rng(Hkv * d + q4)
    for head, tail, budget in [(0, 0, 100), (10, 20, 100), (0, 0, 0), (300, 300, 50), (7, 0, 1), (5, 5, [0, 1, 2, 40, 63, 64, 65, 900, 1500])]:
        r = Rows(rng, [0, 1, 2, 63, 64, 65, 257, 1000, 1500], [3, 0, 1, 2, 0, 0, 5, 0, 1], Hkv, d, q4)
        check(r, head, tail, budget)


@pytest.mark.parametrize("check", [check_in_place, check_away])
@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("n,budget", [(4096, 4095), (4097, 1), (20000, 9000), (20001, 19999), (70000, 333)])
def test_long_requests(n, budget, q4, check):
    H.need_gpu()
    check(Rows(np.random.default_rng(n + budget), [n, 10, n // 3], 2, 1, 64, q4), 16, 33, budget)


@pytest.mark.parametrize("weights", ["equal", "zeros", "special", "negative", "few", "close", "rising", "falling"])
def test_weights_of_every_kind(weights):
    """Ties keep the lower row; NaN is -infinity; -0 is 0."""
    H.need_gpu()
    rng = np.random.default_rng(3)
    n = 5000
    w = {"equal": np.full(n, 0.25), "zeros": np.where(np.arange(n) % 2, 0.0, -0.0),
         "special": rng.choice([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, 1e-45, -1e-45, 3e38], size=n),
         "negative": -rng.random(n), "few": rng.integers(0, 3, size=n), "close": 1.0 + rng.integers(0, 300, size=n) * 2.0 ** -23,
         "rising": np.arange(n), "falling": -np.arange(n)}[weights]
    for budget in (1, 700, 2500, 4999):
        for q4, check in ((True, check_in_place), (False, check_away)):
            check(Rows(rng, [n, 1200], 0, 1, 64, q4, weight=np.tile(w, 2)), 3, 5, budget)


def test_many_requests():
    H.need_gpu()
    rng = np.random.default_rng(4)
    check_in_place(Rows(rng, rng.integers(0, 90, size=1500), 1, 1, 64, True), 2, 3, rng.integers(0, 90, size=1500))


@pytest.mark.parametrize("change,code", [(dict(head=[1, -1, 1]), sonic.ERR_BAD_LAYOUT), (dict(tail=[1, 1, -1]), sonic.ERR_BAD_LAYOUT),
                                         (dict(budget=[-1, 5, 5]), sonic.ERR_BAD_LAYOUT), (dict(length=[-1, 5, 5]), sonic.ERR_BAD_LAYOUT),
                                         (dict(length=[50, 5, 100]), sonic.ERR_BAD_LAYOUT), (dict(cap=[50, 5, 4]), sonic.ERR_CAPACITY),
                                         (dict(status=sonic.ERR_CAPACITY), sonic.ERR_CAPACITY)])
def test_errors_leave_every_request_as_it_was(change, code):
    H.need_gpu()
    rng = np.random.default_rng(5)
    for away in (False, True):
        if "cap" in change and not away:
            continue
        r = Rows(rng, [50, 40, 50], 2, 2, 64, False)
        if "length" in change:
            r.length.copy_(i32(change["length"]))
        r.status.fill_(change.get("status", 0))
        out, _, more = away_cache(r, np.array(change.get("cap", [52, 42, 52])))
        a, kw = r.args(change.get("head", 1), change.get("tail", 1), change.get("budget", 5))
        assert sonic.cache_evict(*a, **kw, **(more if away else {})) == sonic.OK
        torch.cuda.synchronize()
        assert int(r.status.item()) == code
        assert np.array_equal(r.bytes("k"), r.host["k"]) and np.array_equal(r.row_weight.cpu().numpy(), r.weight)
        assert np.array_equal(r.length.cpu().numpy(), change.get("length", r.lens))
        assert torch.all(more["out_len"] == -5) and torch.all(more["out_weight"] == -3.0) and torch.all(out["k"] == 0)


def test_captured_eviction_is_replayed_like_an_eager_one():
    H.need_gpu()
    rng = np.random.default_rng(6)
    r = Rows(rng, [700, 30, 3000], 0, 2, 128, True)
    a, kw = r.args(8, 8, 500)
    start = {n: x.clone() for n, x in r.dev.items()}
    w0, l0 = r.row_weight.clone(), r.length.clone()

    def cycle():
        for n, x in start.items():
            r.dev[n].copy_(x)
        r.row_weight.copy_(w0)
        r.length.copy_(l0)
        assert sonic.cache_evict(*a, **kw) == sonic.OK

    cycle()
    torch.cuda.synchronize()
    want = [x.clone() for x in (*r.dev.values(), r.row_weight, r.length)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cycle()
    for _ in range(4):
        r.row_weight.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (*r.dev.values(), r.row_weight, r.length)))
        cycle()


@pytest.mark.parametrize("q4", [True, False])
def test_rows_past_four_gigabytes(q4):
    H.need_gpu()
    Hkv, d, n, budget = 8, 128, 300, 120
    row = Hkv * d // 2 if q4 else Hkv * d * 2
    first = (1 << 32) // row + 77
    gen = torch.Generator(device="cuda").manual_seed(9)
    shape = [(first + n, Hkv, d // 2), (first + n, Hkv, d // 32)] * 2 if q4 else [(first + n, Hkv, d)] * 2
    planes = [torch.zeros(s, dtype=torch.uint8 if q4 else torch.bfloat16, device="cuda") for s in shape]
    for x in planes:
        x[first:] = torch.randint(0, 200, x[first:].shape, generator=gen, device="cuda").to(x.dtype)
    k, ks, v, vs = planes if q4 else (planes[0], None, planes[1], None)
    w = torch.zeros(first + n, device="cuda")
    w[first:] = torch.rand(n, generator=gen, device="cuda")
    before = [x[first:].clone() for x in planes]
    kept = torch.from_numpy(OE.kept_rows(w[first:].cpu().numpy(), 5, 6, budget)).cuda()
    off, ln, status = torch.tensor([first], dtype=torch.int64, device="cuda"), i32([n]), i32([0])
    ws = torch.zeros(sonic.cache_evict_workspace_bytes(1, n), dtype=torch.uint8, device="cuda")
    lim = (i32([5]), i32([6]), i32([budget]))
    # to another cache, whose rows lie past 4 GiB too, then in place
    out = [torch.zeros_like(x) for x in planes]
    more = dict(k_out=out[0], v_out=out[2 if q4 else 1], out_row_off=off, out_row_cap=i32([n]), out_len=i32([0]), out_weight=torch.zeros_like(w))
    if q4:
        more.update(k_scale_out=out[1], v_scale_out=out[3])
    assert sonic.cache_evict(k, v, off, ln, w, *lim, ws, status, n, k_scale=ks, v_scale=vs, **more) == sonic.OK
    for x, old in zip(out, before):
        assert torch.equal(x[first:first + budget], old[kept]) and not x[:first].any()
    assert sonic.cache_evict(k, v, off, ln, w, *lim, ws, status, n, k_scale=ks, v_scale=vs) == sonic.OK
    for x, old in zip(planes, before):
        assert torch.equal(x[first:first + budget], old[kept]) and torch.equal(x[first + budget:], old[budget:]) and not x[:first].any()
    assert int(ln.item()) == budget and int(status.item()) == 0


# ------------------------------------------------------------------ the prefill's key weights
def test_key_weights_go_to_the_compacted_rows():
    H.need_gpu()
    rng = np.random.default_rng(7)
    lays = [W.random_layout(rng, max_h=4, max_b=300, max_k=90, max_s=60, max_c=60) for _ in range(6)] + [W.RequestLayout(0, [], [], 0)]
    batch = W.make_batch("weights", lays, 4, 2, 64, seed=7)
    db = H.device_batch(batch)
    key_weight = torch.rand(batch.total_tokens, device="cuda")
    caps = H.kept_counts(batch) + 2
    cache = db.alloc_cache(caps)
    assert db.compact() == sonic.OK
    rw = torch.full((cache.k.shape[0],), -1.0, device="cuda")
    call = lambda **c: sonic.kv_compact_weights(**{**dict(cu_seqlens=db.cu, key_weight=key_weight, cache_row_off=cache.row_off,
                                                          cache_len=cache.length, keep_idx=cache.keep_idx, row_weight=rw,
                                                          dev_status=db.status, max_rows=int(caps.max())), **c})
    assert call() == sonic.OK
    assert db.read_status() == 0
    kw, idx, want = key_weight.cpu().numpy(), cache.keep_idx.cpu().numpy(), np.full(len(rw), -1.0, np.float32)
    for b, (o, n) in enumerate(zip(cache.row_off_host, H.kept_counts(batch))):
        want[o:o + n] = kw[batch.cu_seqlens[b] + idx[o:o + n]]
    assert np.array_equal(rw.cpu().numpy(), want)
    # bad calls
    assert call(max_rows=int(cache.length.max()) - 1) == sonic.OK and db.read_status() == sonic.ERR_INVALID_ARG
    db.clear_status()
    assert call(key_weight=key_weight[:-1]) == sonic.OK and db.read_status() == (sonic.ERR_BAD_LAYOUT if lays[5].length else 0)
    db.clear_status()
    for bad in (-1, batch.lengths[0] if hasattr(batch, "lengths") else int(batch.cu_seqlens[1])):
        idx2 = cache.keep_idx.clone()
        idx2[0] = bad
        rw.fill_(-1.0)
        assert call(keep_idx=idx2) == sonic.OK and db.read_status() == sonic.ERR_BAD_LAYOUT
        assert rw[0] == -1.0
        db.clear_status()


# ------------------------------------------------------------------ all of it together
@pytest.mark.parametrize("q4", [True, False])
def test_a_session_from_the_prompt_to_the_next_turn(q4):
    """Prefill with key weights, compaction, weights, eviction to a budget, generation with weights, eviction again, the
    next-turn step over what is left, and a step after it; each part checked against the oracle on what went into it."""
    H.need_gpu()
    rng = np.random.default_rng(8)
    Hq, Hkv, d, steps = 8, 2, 64, 6
    lays = [W.RequestLayout(20, [100, 90], [30, 20], 40), W.RequestLayout(5, [300], [150], 17)]
    batch = W.make_batch("session", lays, Hq, Hkv, d, seed=8, decode_steps=steps + 1)
    db = H.device_batch(batch)
    T, B = batch.total_tokens, 2
    key_weight = torch.zeros(T, device="cuda")
    assert db.prefill(key_weight=key_weight) == sonic.OK
    caps = H.kept_counts(batch) + 30
    cache = db.alloc_cache_q4(caps) if q4 else db.alloc_cache(caps)
    assert (db.compact_q4() if q4 else db.compact()) == sonic.OK
    cache.row_weight = torch.zeros(cache.k.shape[0], device="cuda")
    top = int(caps.max())
    assert sonic.kv_compact_weights(db.cu, key_weight, cache.row_off, cache.length, cache.keep_idx, cache.row_weight, db.status, top) == sonic.OK
    # the oracle's copy: each request's rows as values, and weights
    idx, kw = cache.keep_idx.cpu().numpy(), key_weight.cpu().numpy()
    val = OQ.rounded if q4 else bf16_bits_to_f64
    state = []
    for b, o in enumerate(cache.row_off_host):
        rows = batch.cu_seqlens[b] + idx[o:o + H.kept_counts(batch)[b]]
        state.append([val(batch.k[rows]), val(batch.v[rows]), kw[rows].astype(np.float64)])

    def evict(head, tail, budget):
        got_w = cache.row_weight.cpu().numpy()
        for b, o in enumerate(cache.row_off_host):
            n = len(state[b][0])
            assert np.allclose(got_w[o:o + n], state[b][2], rtol=1e-4, atol=0)     # (weights: see the bars of the decode's tests)
            keep = OE.kept_rows(got_w[o:o + n], head[b], tail[b], budget[b])
            state[b] = [x[keep] for x in state[b]]
        assert cache.evict(i32(head), i32(tail), i32(budget), db.status) == sonic.OK
        assert cache.length.tolist() == [len(s[0]) for s in state]

    def generate(t0, n):
        out = torch.zeros((B, Hq, d), device="cuda")
        for t in range(t0, t0 + n):
            q, k, v = (bf16_to_device(x[t]) for x in (batch.dec_q, batch.dec_k, batch.dec_v))
            st = cache.decode(q, k, v, out, db.status, top, weighted=True) if q4 else cache.decode_weighted(q, k, v, out, db.status, top)
            assert st == sonic.OK
            got = out.cpu().numpy()
            for b in range(B):
                s = state[b]
                s[0], s[1] = (np.concatenate([x, val(new[t, b])[None]]) for x, new in zip(s, (batch.dec_k, batch.dec_v)))
                want, w = OE.attend(batch.dec_q[t, b], s[0], s[1])
                assert np.all(np.abs(got[b] - want) <= 2.0 ** -14 * np.abs(s[1]).max())
                s[2] = np.concatenate([s[2], [0.0]]) + w

    system, current = [20, 5], [40, 17]
    evict(system, current, [80, 60])
    generate(0, steps)
    tail = [c + steps for c in current]
    evict(system, tail, [75, 50])
    assert db.read_status() == 0
    # the turn's rows get three Nexus rows over what the eviction left
    keep = [len(s[0]) - t for s, t in zip(state, tail)]
    nq, nk, nv = (W.f32_to_bf16_bits(rng.standard_normal((6, h, d)).astype(np.float32)) for h in (Hq, Hkv, Hkv))
    wide = CompactCache(int(caps.sum()), Hkv, d, cache.row_off_host, cache.row_cap_host, "cuda") if q4 else cache
    if q4:
        assert cache.expand(i32([0, 0]), cache.length, wide.k, wide.v, wide.row_off, wide.row_cap, db.status, top) == sonic.OK
        wide.length.copy_(cache.length)
    out = torch.zeros((6, Hq, d), device="cuda")
    ws = torch.zeros(sonic.nexus_extend_workspace_bytes(B, 6, top, Hkv, d), dtype=torch.uint8, device="cuda")
    assert sonic.nexus_extend(i32([0, 3, 6]), i32(keep), wide.k, wide.v, wide.row_off, wide.row_cap, wide.length, bf16_to_device(nq),
                              bf16_to_device(nk), bf16_to_device(nv), out, ws, db.status, top) == sonic.OK
    got = out.cpu().numpy()
    for b in range(B):
        rows = slice(3 * b, 3 * b + 3)
        k, v = (np.concatenate([x, bf16_bits_to_f64(new[rows])]) for x, new in zip(state[b], (nk, nv)))
        want = np.stack([OE.attend(x, k, v)[0] for x in nq[rows]])
        H.assert_close(got[rows], want, f"next turn, request {b}")
        state[b] = [np.concatenate([x[:keep[b]], val(new[rows])]) for x, new in zip(state[b], (nk, nv))] + [
            np.concatenate([state[b][2][:keep[b]], np.zeros(3)])]
    if q4:   # back to 4 bits: the cache as a packed batch, the rows past each length as text
        n = wide.length.tolist()
        role = np.full(int(caps.sum()), 1, np.uint8)
        for o, m in zip(cache.row_off_host, n):
            role[o:o + m] = 3
        cu = i32(np.concatenate([[0], np.cumsum(caps)]))
        assert sonic.kv_compact_q4(cu, torch.from_numpy(role).cuda(), wide.k, wide.v, cache.k, cache.k_scale, cache.v, cache.v_scale,
                                   cache.row_off, cache.row_cap, cache.length, cache.keep_idx, db.status, top) == sonic.OK
        assert cache.length.tolist() == n
    for b, o in enumerate(cache.row_off_host):
        cache.row_weight[int(o) + keep[b]:int(o) + keep[b] + 3] = 0.0
    generate(steps, 1)
    assert db.read_status() == 0
