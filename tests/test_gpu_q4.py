"""The 4-bit cache on the GPU against the oracles: rows bit for bit, attention and weights within bars counted from
the roundings on the way.

Bars.  A decode output is a convex combination of V values whose probabilities are off by a relative EPS = 2^-15:
the bf16 parts of a probability leave 2^-17 of it at most, the exponential of a 32-bit score of log2 size up to 64 is off
by 64 * 2^-24 / log2(e) and the hardware's 2^-22, and sums of 32-bit values add less; the sum of the probabilities is
off by as much again.  So |out - exact| <= 2 * EPS * max|V|, and a weight, a mean of such probabilities, is within
2 * EPS of itself and half a step of the sum it is added to.
"""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import compaction as OC
from oracle import evict as OE
from oracle import q4 as OQ
from oracle.attention import bf16_bits_to_f64
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import CompactCache, Q4Cache, bf16_to_device, bf16_to_host
from tests import gpu_helpers as H

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -15
HEADS = [(4, 2, 64), (8, 1, 64), (28, 4, 128), (32, 8, 128), (5, 5, 64), (6, 3, 128), (21, 7, 128), (12, 2, 64), (5, 1, 128),
         (40, 8, 64), (3, 1, 128)]


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def normal_bits(rng, *shape, scale=1.0):
    return W.f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


class Cache:
    """A cache of given lengths on both sides: bf16 or 4-bit rows, weights, and the values each row stands for."""

    def __init__(self, rng, lens, extra, Hkv, d, q4, fill=None):
        self.lens, self.Hkv, self.d, self.q4 = np.asarray(lens), Hkv, d, q4
        cap = self.lens + extra
        off = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
        n = int(cap.sum())
        self.dev = (Q4Cache if q4 else CompactCache)(n, Hkv, d, off, cap, "cuda")
        channel = np.exp(0.7 * rng.standard_normal((1, Hkv, d)))
        self.bits = [normal_bits(rng, n, Hkv, d, scale=channel) for _ in range(2)]
        self.values = [OQ.rounded(x) if q4 else bf16_bits_to_f64(x) for x in self.bits]
        valid = np.zeros(n, bool)
        for o, m in zip(off, lens):
            valid[o:o + m] = True
        for x, bits in ((self.dev.k, self.bits[0]), (self.dev.v, self.bits[1])):
            if q4:
                codes, scales = OQ.encode(bits)
                s = self.dev.k_scale if x is self.dev.k else self.dev.v_scale
                x[torch.from_numpy(valid)] = torch.from_numpy(OQ.pack(codes)[valid]).cuda()
                s[torch.from_numpy(valid)] = torch.from_numpy(scales[valid]).cuda()
            else:
                x[torch.from_numpy(valid)] = bf16_to_device(bits[valid])
        self.dev.length.copy_(i32(lens))
        self.weight = rng.random(n).astype(np.float32)
        self.dev.row_weight = torch.from_numpy(self.weight).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.off, self.cap, self.max_ctx = off, cap, int(cap.max())

    def step(self, rng, Hq, weighted=True, max_ctx=None, scale=1.0):
        """One step's inputs and outputs."""
        B = len(self.lens)
        q, k, v = (normal_bits(rng, B, h, self.d, scale=s) for h, s in ((Hq, scale), (self.Hkv, 1), (self.Hkv, 1)))
        out = torch.full((B, Hq, self.d), 7.0, device="cuda")
        args = (bf16_to_device(q), bf16_to_device(k), bf16_to_device(v), out, self.status, max_ctx or self.max_ctx)
        if self.q4:
            st = self.dev.decode(*args, weighted=weighted)
        else:
            st = self.dev.decode_weighted(*args)
        assert st == sonic.OK, sonic.status_string(st)
        torch.cuda.synchronize()
        return q, k, v, out.cpu().numpy()

    def expect(self, b, q, k, v):
        """The oracle's step for request b; its row is appended on the oracle's side too."""
        o, n = int(self.off[b]), int(self.lens[b])
        for x, new in zip(self.values, (k, v)):
            x[o + n] = OQ.rounded(new[b]) if self.q4 else bf16_bits_to_f64(new[b])
        return OE.attend(q[b], self.values[0][o:o + n + 1], self.values[1][o:o + n + 1])

    def check(self, q, k, v, out, weighted=True, skip=()):
        B = len(self.lens)
        got_w = self.dev.row_weight.cpu().numpy()
        for b in range(B):
            if b in skip:
                continue
            o, n = int(self.off[b]), int(self.lens[b])
            want, w = self.expect(b, q, k, v)
            top = np.abs(self.values[1][o:o + n + 1]).max()
            assert np.all(np.abs(out[b] - want) <= 2 * EPS * top), (b, n, np.abs(out[b] - want).max() / top)
            if weighted:
                full = w + np.concatenate([self.weight[o:o + n].astype(np.float64), [0.0]])
                assert np.all(np.abs(got_w[o:o + n + 1] - full) <= 2 * EPS * w + 2.0 ** -24 * full), b
                self.weight[o:o + n + 1] = got_w[o:o + n + 1]
            self.lens[b] += 1
        assert np.array_equal(got_w, self.weight)     # every other row's weight is as it was
        assert np.array_equal(self.dev.length.cpu().numpy(), self.lens)


# ------------------------------------------------------------------ rows
def compact(k, v, role, cu, cap, Hkv, d):
    cap = np.asarray(cap)
    off = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
    c = Q4Cache(int(cap.sum()), Hkv, d, off, cap, "cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    st = sonic.kv_compact_q4(i32(cu), torch.from_numpy(role).cuda(), bf16_to_device(k), bf16_to_device(v), c.k, c.k_scale, c.v, c.v_scale,
                             c.row_off, c.row_cap, c.length, c.keep_idx, status, int(np.diff(cu).max()))
    assert st == sonic.OK
    torch.cuda.synchronize()
    return c, int(status.item())


def test_every_bf16_value_is_rounded_as_defined():
    """Blocks of 32 neighbouring patterns, and every eighth pattern above fractions of itself at and around the borders."""
    H.need_gpu()
    runs = np.arange(65536, dtype=np.uint16).reshape(-1, 32)
    top = np.arange(0, 65536, 8, dtype=np.uint16)
    with np.errstate(all="ignore"):
        f = bf16_bits_to_f64(top)
        parts = np.concatenate([np.arange(1, 16) / 16, np.arange(1, 15) / 14, [0.0078125, 0.03]])
        below = W.f32_to_bf16_bits(np.where(np.isfinite(f), f, 1.0)[:, None] * parts * np.where(np.arange(31) % 3, 1, -1))
    blocks = np.concatenate([runs, np.concatenate([top[:, None], below], 1)])
    k = blocks.reshape(-1, 1, 64)
    v = k[::-1].copy()
    c, status = compact(k, v, np.full(len(k), 3, np.uint8), [0, len(k)], [len(k)], 1, 64)
    assert status == 0
    for bits, codes, scales in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        wc, ws = OQ.encode(bits)
        assert np.array_equal(scales.cpu().numpy(), ws)
        assert np.array_equal(codes.cpu().numpy(), OQ.pack(wc))
    out = torch.zeros((2,) + k.shape, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert c.expand(i32([0]), c.length, out[0], out[1], c.row_off, c.row_cap, status, len(k)) == sonic.OK
    for got, bits in zip(out.double().cpu().numpy(), (k, v)):
        assert np.array_equal(got, OQ.rounded(bits), equal_nan=True)


@pytest.mark.parametrize("seed,Hkv,d", [(1, 2, 64), (2, 8, 128), (3, 1, 128), (4, 5, 64), (5, 3, 128), (6, 1, 64)])
def test_compaction_rows_and_lengths(seed, Hkv, d):
    H.need_gpu()
    rng = np.random.default_rng(seed)
    lays = [W.random_layout(rng, max_h=5, max_b=700, max_k=200, max_s=300, max_c=300) for _ in range(5)]
    lays += [W.RequestLayout(0, [], [], 0), W.RequestLayout(0, [3000], [0], 0), W.RequestLayout(0, [3000], [1], 0)]
    batch = W.make_batch("q4", lays, Hkv, Hkv, d, seed=seed, scales=True)
    cap = H.kept_counts(batch) + rng.integers(0, 40, size=len(lays))
    c, status = compact(batch.k, batch.v, batch.role, batch.cu_seqlens, cap, Hkv, d)
    assert status == 0
    kc, vc, idx, n, off = H.oracle_compact(batch, cap)
    assert np.array_equal(c.length.cpu().numpy(), n) and np.array_equal(c.keep_idx.cpu().numpy(), idx)
    kept = idx >= 0
    for bits, codes, scales in ((kc, c.k, c.k_scale), (vc, c.v, c.v_scale)):
        wc, ws = OQ.encode(bits[kept])
        assert np.array_equal(codes.cpu().numpy()[kept], OQ.pack(wc)) and np.array_equal(scales.cpu().numpy()[kept], ws)
        assert np.all(codes.cpu().numpy()[~kept] == 255) and np.all(scales.cpu().numpy()[~kept] == 255)


def test_compaction_capacity_and_expand_errors():
    H.need_gpu()
    rng = np.random.default_rng(7)
    k = normal_bits(rng, 60, 2, 64)
    role = np.full(60, 3, np.uint8)
    c, status = compact(k, k, role, [0, 40, 60], [39, 20], 2, 64)
    assert status == sonic.ERR_CAPACITY and int(c.length[0]) == 0
    assert np.all(c.k.cpu().numpy()[39:] == OQ.pack(OQ.encode(k[40:])[0])) or np.all(c.k.cpu().numpy()[39:] == 255)
    c, status = compact(k, k, role, [0, 40, 60], [40, 20], 2, 64)
    out = torch.zeros((2, 60, 2, 64), dtype=torch.bfloat16, device="cuda")
    for begin, end, cap, max_rows, code in [([0, -1], [3, 3], [40, 20], 40, sonic.ERR_BAD_LAYOUT), ([0, 4], [3, 3], [40, 20], 40, sonic.ERR_BAD_LAYOUT),
                                            ([0, 0], [3, 21], [40, 20], 40, sonic.ERR_BAD_LAYOUT), ([0, 0], [3, 20], [40, 19], 40, sonic.ERR_CAPACITY),
                                            ([0, 0], [3, 20], [40, 20], 19, sonic.ERR_INVALID_ARG)]:
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        out.fill_(5.0)
        assert c.expand(i32(begin), i32(end), out[0], out[1], c.row_off, i32(cap), st, max_rows) == sonic.OK
        assert int(st.item()) == code
        assert torch.all(out[:, 40:] == 5.0)                                   # nothing of the request at fault
        assert c.expand(i32([0, 0]), i32([3, 3]), out[0], out[1], c.row_off, c.row_cap, st, 40) == sonic.OK
        assert torch.all(out[:, 40:] == 5.0)                                   # a pending status stops the call


def test_expand_ranges_leave_other_rows():
    H.need_gpu()
    rng = np.random.default_rng(8)
    c = Cache(rng, [50, 0, 700, 1], 3, 3, 128, True)
    begin, end = [10, 0, 1, 0], [11, 0, 700, 1]
    out = torch.full((2, 1000, 3, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([900, 3, 100, 0], dtype=torch.int64, device="cuda")
    assert c.dev.expand(i32(begin), i32(end), out[0], out[1], off, i32([1, 0, 699, 1]), c.status, 699) == sonic.OK
    assert int(c.status.item()) == 0
    got = out.double().cpu().numpy()
    for x, values in zip(got, c.values):
        touched = np.zeros(1000, bool)
        for b, dst in enumerate([900, 3, 100, 0]):
            n, o = end[b] - begin[b], int(c.off[b]) + begin[b]
            assert np.array_equal(x[dst:dst + n], values[o:o + n])
            touched[dst:dst + n] = True
        assert np.all(x[~touched] == 5.0)


# ------------------------------------------------------------------ decode
@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_decode_steps(Hq, Hkv, d, q4):
    H.need_gpu()
    rng = np.random.default_rng(Hq * 1000 + d + q4)
    c = Cache(rng, [0, 1, 15, 16, 17, 255, 333, 600], 3, Hkv, d, q4)
    for _ in range(3):
        step = c.step(rng, Hq)
        assert int(c.status.item()) == 0
        c.check(*step)
    if q4:   # the appended rows, bit for bit
        for b in range(len(c.lens)):
            rows = slice(int(c.off[b] + c.lens[b]) - 3, int(c.off[b] + c.lens[b]))
            got = OQ.decode(OQ.unpack(c.dev.k[rows].cpu().numpy()), c.dev.k_scale[rows].cpu().numpy())
            assert np.array_equal(got, c.values[0][rows])
            got = OQ.decode(OQ.unpack(c.dev.v[rows].cpu().numpy()), c.dev.v_scale[rows].cpu().numpy())
            assert np.array_equal(got, c.values[1][rows])


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("lens,Hq,Hkv,d", [([9000], 8, 2, 128), ([40000], 2, 1, 64), ([5000, 3], 7, 1, 128), ([2500, 10, 700, 4000] * 2, 8, 8, 64),
                                           ([16500], 8, 8, 128), ([33000], 4, 4, 64)])
def test_decode_long_contexts(lens, Hq, Hkv, d, q4):
    """Contexts cut into many ranges, and several lengths in one call."""
    H.need_gpu()
    rng = np.random.default_rng(sum(lens) + q4)
    c = Cache(rng, lens, 2, Hkv, d, q4)
    for _ in range(2):
        c.check(*c.step(rng, Hq))


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("B,Hq,Hkv,d,top", [(64, 8, 4, 64, 2300), (40, 8, 8, 128, 2100), (64, 28, 4, 128, 2048), (33, 16, 8, 64, 400), (300, 4, 1, 64, 90),
                                             (130, 8, 8, 64, 200)])
def test_decode_many_requests(B, Hq, Hkv, d, top, q4):
    """256 and more pairs: one range a pair, and rows shared over the batch."""
    H.need_gpu()
    rng = np.random.default_rng(B + top + q4)
    lens = np.maximum(0, (top * rng.random(B) ** 3).astype(int))
    lens[1] = top
    c = Cache(rng, lens, 2, Hkv, d, q4)
    for _ in range(2):
        c.check(*c.step(rng, Hq))


@pytest.mark.parametrize("q4", [True, False])
def test_a_bound_far_above_the_lengths(q4):
    """Most ranges of the grid have no rows; then shared rows with more workgroups than ranges."""
    H.need_gpu()
    rng = np.random.default_rng(21 + q4)
    for lens, Hq, Hkv in (([3, 40, 0, 300], 4, 2), ([5] * 50, 8, 8)):
        c = Cache(rng, lens, 2, Hkv, 64, q4)
        for _ in range(2):
            c.check(*c.step(rng, Hq, max_ctx=9000))


def test_no_tokens_at_all():
    H.need_gpu()
    k = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    c = Q4Cache(4, 2, 64, np.array([0, 2]), np.array([2, 2]), "cuda")
    c.length.fill_(9)
    status = i32([0])
    assert sonic.kv_compact_q4(i32([0, 0, 0]), torch.zeros(0, dtype=torch.uint8, device="cuda"), k, k, c.k, c.k_scale, c.v, c.v_scale, c.row_off,
                               c.row_cap, c.length, c.keep_idx, status, 0) == sonic.OK
    assert c.length.tolist() == [0, 0] and int(status.item()) == 0 and torch.all(c.k == 255)


def test_decode_without_weights_gives_the_same_outputs():
    H.need_gpu()
    outs = []
    for weighted in (True, False):
        rng = np.random.default_rng(5)
        c = Cache(rng, [700, 20, 3000], 2, 2, 128, True)
        outs.append(c.step(rng, 8, weighted=weighted)[3])
        if not weighted:
            assert np.array_equal(c.dev.row_weight.cpu().numpy(), c.weight)
    assert np.array_equal(outs[0], outs[1])


@pytest.mark.parametrize("q4", [True, False])
def test_full_requests_and_pending_errors(q4):
    H.need_gpu()
    rng = np.random.default_rng(11)
    c = Cache(rng, [30, 300, 5], 1, 2, 64, q4)
    c.check(*c.step(rng, 4))
    # all are full now
    before = c.dev.row_weight.clone()
    *_, out = c.step(rng, 4)
    assert int(c.status.item()) == sonic.ERR_CAPACITY
    assert np.all(out == 7.0) and torch.equal(before, c.dev.row_weight) and np.array_equal(c.dev.length.cpu().numpy(), c.lens)
    # one of them full: the others go on, a pending capacity error does not stop them
    c = Cache(rng, [30, 300, 5], 2, 2, 64, q4)
    c.dev.row_cap.copy_(i32([32, 300, 7]))
    for _ in range(2):
        step = c.step(rng, 4)
        assert int(c.status.item()) == sonic.ERR_CAPACITY and np.all(step[3][1] == 7.0)
        c.check(*step, skip=(1,))
    # another pending error stops the call
    c.status.fill_(sonic.ERR_BAD_LAYOUT)
    before = c.dev.row_weight.clone()
    *_, out = c.step(rng, 4)
    assert np.all(out == 7.0) and torch.equal(before, c.dev.row_weight) and np.array_equal(c.dev.length.cpu().numpy(), c.lens)
    c.status.zero_()
    c = Cache(rng, [30, 31], 2, 2, 64, q4)
    c.check(*c.step(rng, 4))


def test_full_requests_where_rows_are_shared():
    H.need_gpu()
    rng = np.random.default_rng(12)
    lens = np.full(64, 60)
    lens[3] = 2100
    c = Cache(rng, lens, 2, 4, 64, True)
    cap = c.cap.copy()
    cap[[0, 5]] = lens[[0, 5]]
    c.dev.row_cap.copy_(i32(cap))
    step = c.step(rng, 4)
    assert int(c.status.item()) == sonic.ERR_CAPACITY
    c.check(*step, skip=(0, 5))
    c.dev.row_cap.copy_(i32(c.lens))            # all full
    before = c.dev.row_weight.clone()
    *_, out = c.step(rng, 4)
    assert np.all(out == 7.0) and torch.equal(before, c.dev.row_weight)


def test_infinities_and_nan_reach_only_what_they_should():
    H.need_gpu()
    rng = np.random.default_rng(13)
    c = Cache(rng, [40, 40, 400], 2, 2, 128, True)
    q, k, v = (normal_bits(rng, 3, h, 128) for h in (4, 2, 2))
    v[0, 1, 70], k[1, 0, 5] = 0x7F80, 0x7FC0
    out = torch.zeros((3, 4, 128), device="cuda")
    assert c.dev.decode(bf16_to_device(q), bf16_to_device(k), bf16_to_device(v), out, c.status, c.max_ctx, weighted=True) == sonic.OK
    nan = np.isnan(out.cpu().numpy())
    want = np.zeros_like(nan)
    want[0, 2:, 64:96] = True      # the block of V that held the infinity, for the q-heads of its kv-head
    want[1, :2] = True             # a NaN score
    assert np.array_equal(nan, want)
    w = c.dev.row_weight.cpu().numpy()
    assert np.isnan(w[42:42 + 41]).all() and not np.isnan(np.delete(w, range(42, 42 + 41))).any()


@pytest.mark.parametrize("q4", [True, False])
def test_a_nan_key_in_one_range_makes_every_weight_nan(q4):
    """The range holds nothing but NaN scores: its maximum is none, and it still counts."""
    H.need_gpu()
    rng = np.random.default_rng(14)
    c = Cache(rng, [2048], 2, 1, 64, q4)
    if q4:
        c.dev.k_scale[200:900] = 255
    else:
        c.dev.k[200:900] = float("nan")
    *_, out = c.step(rng, 2)
    assert np.isnan(out).all()
    assert np.isnan(c.dev.row_weight.cpu().numpy()[:2049]).all()


@pytest.mark.parametrize("q4", [True, False])
def test_large_scores(q4):
    """Scores of several hundred: one row takes all, and the others' weights are exactly the exponentials'."""
    H.need_gpu()
    rng = np.random.default_rng(15)
    c = Cache(rng, [500, 3], 2, 2, 64, q4)
    q, k, v, out = c.step(rng, 4, scale=50.0)
    for b in range(2):
        o, n = int(c.off[b]), int(c.lens[b])
        want, _ = c.expect(b, q, k, v)
        # scores up to 2^11 in log2 units are off by 2^11 * 2^-22 with their sums of 64 products
        assert np.all(np.abs(out[b] - want) <= 2.0 ** -10 * np.abs(c.values[1][o:o + n + 1]).max())


def test_captured_steps_are_replayed_like_eager_ones():
    H.need_gpu()
    rng = np.random.default_rng(16)
    steps, Hq = 3, 8
    c = Cache(rng, [100, 900, 17], 2 * steps, 2, 128, True)
    B = len(c.lens)
    q, k, v = (bf16_to_device(normal_bits(rng, steps, B, h, 128)) for h in (Hq, 2, 2))
    out = torch.zeros((steps, B, Hq, 128), device="cuda")
    start, w0 = c.dev.length.clone(), c.dev.row_weight.clone()

    def loop():
        torch.add(start, 0, out=c.dev.length)
        torch.add(w0, 0, out=c.dev.row_weight)
        for t in range(steps):
            assert c.dev.decode(q[t], k[t], v[t], out[t], c.status, c.max_ctx, weighted=True) == sonic.OK

    loop()
    torch.cuda.synchronize()
    want, want_w = out.clone(), c.dev.row_weight.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loop()
    for _ in range(4):
        out.zero_()
        c.dev.row_weight.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(c.dev.row_weight, want_w) and torch.equal(c.dev.length, start + steps)
        loop()                        # eager work in between
        assert torch.equal(out, want)
    assert int(c.status.item()) == 0


def test_steps_on_a_stream_of_their_own():
    H.need_gpu()
    rng = np.random.default_rng(17)
    c = Cache(rng, [100, 900], 2, 2, 64, True)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        step = c.step(rng, 8)
    c.check(*step)


def test_a_status_word_that_changes_while_calls_run_leaves_the_next_call_right():
    H.need_gpu()
    rng = np.random.default_rng(18)
    c = Cache(rng, [100, 900, 3000, 5], 40, 2, 64, True)
    flips = H.Flips(c.status, sonic.ERR_BAD_LAYOUT)
    B = 4
    q, k, v = (bf16_to_device(normal_bits(rng, B, h, 64)) for h in (4, 2, 2))
    out = torch.zeros((B, 4, 64), device="cuda")
    flips.start()
    for _ in range(20):
        assert c.dev.decode(q, k, v, out, c.status, c.max_ctx, weighted=True) == sonic.OK
    torch.cuda.synchronize()
    c.status.zero_()
    c.dev.length.copy_(i32(c.lens))
    c.dev.row_weight.copy_(torch.from_numpy(c.weight))
    c.check(*c.step(rng, 4))


def test_rows_past_four_gigabytes():
    """Codes, scales and bf16 rows behind the first 4 GiB of their tensors: compaction, step, reading back."""
    H.need_gpu()
    rng = np.random.default_rng(20)
    Hkv, d, n = 8, 128, 70
    first = (1 << 32) // (Hkv * d // 2) + 1000          # of the codes
    k, v = normal_bits(rng, n, Hkv, d), normal_bits(rng, n, Hkv, d)
    off = torch.tensor([first], dtype=torch.int64, device="cuda")
    planes = [torch.full((first + n + 1, Hkv, w), 255, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32, d // 2, d // 32)]
    kc, ks, vc, vs = planes
    idx, ln, status = torch.zeros(first + n + 1, dtype=torch.int32, device="cuda"), i32([0]), i32([0])
    cap = i32([n + 1])
    assert sonic.kv_compact_q4(i32([0, n]), torch.full((n,), 3, dtype=torch.uint8, device="cuda"), bf16_to_device(k), bf16_to_device(v), kc, ks,
                               vc, vs, off, cap, ln, idx, status, n) == sonic.OK
    q, kn, vn = (normal_bits(rng, 1, h, d) for h in (16, Hkv, Hkv))
    out = torch.zeros((1, 16, d), device="cuda")
    weight = torch.zeros(first + n + 1, device="cuda")
    ws = torch.zeros(sonic.decode_q4_workspace_bytes(1, 16, d, n + 1, True), dtype=torch.uint8, device="cuda")
    assert sonic.compressed_decode_q4(kc, ks, vc, vs, off, cap, ln, bf16_to_device(q), bf16_to_device(kn), bf16_to_device(vn), out, ws, status,
                                      n + 1, row_weight=weight) == sonic.OK
    kv = [OQ.rounded(np.concatenate(x)) for x in ((k, kn), (v, vn))]
    want, w = OE.attend(q[0], *kv)
    assert int(status.item()) == 0 and int(ln.item()) == n + 1
    assert np.all(np.abs(out[0].cpu().numpy() - want) <= 2 * EPS * np.abs(kv[1]).max())
    assert np.all(np.abs(weight[first:].cpu().numpy() - w) <= 2 * EPS * w) and not weight[:first].any()
    assert torch.all(kc[:first] == 255) and torch.all(vs[:first] == 255)
    # back to bf16 rows that lie past 4 GiB too
    far = (1 << 32) // (Hkv * d * 2) + 10
    ko, vo = (torch.zeros((far + n + 1, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert sonic.cache_expand_q4(kc, ks, vc, vs, off, cap, i32([0]), ln, ko, vo, torch.tensor([far], dtype=torch.int64, device="cuda"), cap,
                                 status, n + 1) == sonic.OK
    for got, values in ((ko, kv[0]), (vo, kv[1])):
        assert np.array_equal(got[far:].double().cpu().numpy(), values) and not got[:far].any()


def test_binding_refusals():
    H.need_gpu()
    rng = np.random.default_rng(19)
    c = Cache(rng, [10, 12], 2, 2, 64, True)
    d = c.dev
    q, k, out = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda"), \
        torch.zeros((2, 4, 64), device="cuda")
    ws = torch.zeros(sonic.decode_q4_workspace_bytes(2, 4, 64, 14, True), dtype=torch.uint8, device="cuda")
    good = dict(k_cache=d.k, k_scale=d.k_scale, v_cache=d.v, v_scale=d.v_scale, cache_row_off=d.row_off, cache_row_cap=d.row_cap,
                cache_len=d.length, q=q, k_new=k, v_new=k, out=out, workspace=ws, dev_status=c.status, max_ctx=14, row_weight=d.row_weight)
    assert sonic.compressed_decode_q4(**good) == sonic.OK
    for name, bad in [("k_scale", d.v), ("k_cache", d.k[:, :1]), ("row_weight", d.row_weight[:-1]), ("cache_len", d.length[:1]),
                      ("out", out[:, :2].contiguous()), ("k_new", k[:1])]:
        with pytest.raises(ValueError):
            sonic.compressed_decode_q4(**{**good, name: bad})
    for name, bad in [("row_weight", d.row_weight.double()), ("q", q.half()), ("k_cache", d.k.to(torch.int32))]:
        with pytest.raises(TypeError):
            sonic.compressed_decode_q4(**{**good, name: bad})
    assert sonic.compressed_decode_q4(**{**good, "workspace": ws[:256]}) == sonic.ERR_WORKSPACE
