"""The attention of drafted tokens on the GPU against the 64-bit oracle, within bars counted from the roundings on the way.

Bars.  An output is a convex combination of V values.  fp32: its probabilities are off by a relative EPS = 2^-15 at most
(their three bf16 parts leave 2^-26, the exponential of a 32-bit score of log2 size up to 64 is off by 64 * 2^-24 / log2(e)
and the hardware's 2^-22, and sums of 32-bit values add less), and so is their sum: |out - exact| <= 2 * EPS * max|V|.
bf16: a probability is rounded to bf16, by 2^-8 of it at most, and so is their sum, and the output is rounded once more:
|out - exact| <= (3 * 2^-8 + 2 * EPS) * max|V|, and 2^-15 of that for the products of two such terms.
"""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import q4 as OQ
from oracle import tree as OT
from oracle.attention import bf16_bits_to_f64
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import DraftStep, bf16_to_device
from tests import gpu_helpers as H
from tests.test_gpu_q4 import EPS, HEADS, Cache, i32, normal_bits

pytestmark = pytest.mark.gpu

BAR = {"fp32": 2 * EPS, "bf16": (3 * 2.0 ** -8 + 2 * EPS) * 1.01}
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def tree(rng, n, kind="bushy"):
    if kind == "chain":
        return np.arange(n) - 1
    if kind == "star":
        return np.where(np.arange(n) == 0, -1, 0)
    if kind == "forest":
        return np.array([-1 if rng.random() < 0.3 else rng.integers(-1, i) for i in range(n)], int)
    return np.array([-1] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, n)], int)[:n]


class Step:
    """One call's inputs on both sides."""

    def __init__(self, rng, cache, Hq, nodes, kind="bushy", spare=0, scale=1.0):
        self.c, self.nodes = cache, nodes
        self.parents = [tree(rng, n, kind) for n in nodes]
        self.cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        self.N = int(self.cu[-1]) + spare
        self.q = normal_bits(rng, self.N, Hq, cache.d, scale=scale)
        self.k, self.v = (normal_bits(rng, self.N, cache.Hkv, cache.d) for _ in range(2))
        self.step = DraftStep(len(nodes), self.N, max(max(nodes), 1))
        flat = np.concatenate(self.parents + [np.zeros(spare, int)])
        self.parent = None if kind == "chain" else i32(flat)
        self.status = cache.status
        self.max_ctx = int(max(cache.lens))

    def run(self, out="fp32", max_ctx=None, stream=None, plan=True):
        got = torch.full((self.N,) + self.q.shape[1:], 7.0, dtype=DTYPE[out], device="cuda")
        if plan:
            assert self.step.plan_trees(i32(self.cu), self.parent, self.status, stream=stream) == sonic.OK
        st = self.c.dev.tree_decode(self.step.plan, *(bf16_to_device(x) for x in (self.q, self.k, self.v)), got, self.status,
                                    self.step.max_nodes, self.max_ctx if max_ctx is None else max_ctx, stream=stream)
        assert st == sonic.OK, sonic.status_string(st)
        torch.cuda.synchronize()
        return got.double().cpu().numpy()

    def expect(self, b):
        c, s, e = self.c, self.cu[b], self.cu[b + 1]
        o, n = int(c.off[b]), int(c.lens[b])
        k, v = ((OQ.rounded(x[s:e]) if c.q4 else bf16_bits_to_f64(x[s:e])) for x in (self.k, self.v))
        with np.errstate(invalid="ignore"):
            want = OT.attend(bf16_bits_to_f64(self.q[s:e]), c.values[0][o:o + n], c.values[1][o:o + n], k, v, self.parents[b])
        seen = np.concatenate([c.values[1][o:o + n], v])
        return want, np.abs(seen[np.isfinite(seen)]).max() if seen.size else 0.0

    def check(self, got, out="fp32", skip=()):
        assert int(self.status.item()) == 0 or skip
        for b in range(len(self.nodes)):
            if b in skip or self.nodes[b] == 0:
                continue
            want, top = self.expect(b)
            err = np.abs(got[self.cu[b]:self.cu[b + 1]] - want)
            assert np.all(err <= BAR[out] * top), (b, self.c.lens[b], self.nodes[b], err.max() / top)
        assert np.all(got[self.cu[-1]:] == 7.0)          # rows behind the last request


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_trees(Hq, Hkv, d, q4, out):
    """Lengths and node counts around the blocks of 32, empty caches, requests without nodes, rows behind the last."""
    H.need_gpu()
    rng = np.random.default_rng(Hq * 1000 + d + q4)
    c = Cache(rng, [0, 1, 31, 32, 33, 255, 333, 600, 40], 1, Hkv, d, q4)
    for nodes in ([1, 5, 4, 1, 2, 3, 1, 5, 0], [7, 0, 33, 3, 32, 1, 31, 12, 9]):
        s = Step(rng, c, Hq, nodes, spare=3)
        s.check(s.run(out), out)


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("kind", ["chain", "star", "forest", "bushy"])
def test_large_trees_of_every_kind(kind, q4, out):
    H.need_gpu()
    rng = np.random.default_rng(len(kind) + q4)
    c = Cache(rng, [70, 0, 500], 1, 2, 64, q4)
    s = Step(rng, c, 6, [256, 129, 64], kind)
    s.check(s.run(out), out)


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,d,nodes", [([9000], 8, 2, 128, [9]), ([40000], 2, 1, 64, [3]), ([5000, 3], 7, 1, 128, [2, 30]),
                                                 ([2500, 10, 700, 4000] * 2, 8, 8, 64, [1] * 8), ([16500], 8, 8, 128, [17]),
                                                 ([3000, 1], 4, 4, 64, [100, 3])])
def test_long_contexts(lens, Hq, Hkv, d, nodes, q4):
    """Requests cut into many ranges, and several lengths in one call."""
    H.need_gpu()
    rng = np.random.default_rng(sum(lens) + q4)
    s = Step(rng, Cache(rng, lens, 1, Hkv, d, q4), Hq, nodes)
    for out in ("fp32", "bf16"):
        s.check(s.run(out), out)


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,d,top", [(64, 8, 4, 64, 900), (300, 4, 1, 64, 90), (33, 16, 8, 64, 400)])
def test_many_requests(B, Hq, Hkv, d, top, q4):
    H.need_gpu()
    rng = np.random.default_rng(B + top + q4)
    lens = np.maximum(0, (top * rng.random(B) ** 3).astype(int))
    lens[1] = top
    s = Step(rng, Cache(rng, lens, 1, Hkv, d, q4), Hq, [int(x) for x in rng.integers(0, 7, B)])
    s.check(s.run("fp32"), "fp32")


@pytest.mark.parametrize("q4", [False, True])
def test_a_bound_far_above_the_lengths(q4):
    H.need_gpu()
    rng = np.random.default_rng(21 + q4)
    s = Step(rng, Cache(rng, [3, 40, 0, 300], 1, 2, 64, q4), 4, [3, 1, 2, 4])
    whole = s.run(max_ctx=300)
    s.check(whole)
    s.check(s.run(max_ctx=90000))


def test_one_node_is_a_decode_step():
    """Without its append: what the decode over the same cache gives."""
    H.need_gpu()
    for q4 in (False, True):
        rng = np.random.default_rng(5 + q4)
        c = Cache(rng, [700, 20, 3000], 1, 2, 128, q4)
        s = Step(rng, c, 8, [1, 1, 1])
        got = s.run()
        s.check(got)
        out = torch.empty((3, 8, 128), device="cuda")
        args = [bf16_to_device(x) for x in (s.q, s.k, s.v)] + [out, c.status, c.max_ctx]
        assert (c.dev.decode(*args) if q4 else c.dev.decode_weighted(*args)) == sonic.OK
        top = max(np.abs(c.values[1]).max(), np.abs(bf16_bits_to_f64(s.v)).max())
        assert np.abs(out.double().cpu().numpy() - got).max() <= 4 * EPS * top


def test_softmax_scale_and_large_scores():
    """Scores of several hundred; and a range whose every score lies far below another's."""
    H.need_gpu()
    rng = np.random.default_rng(9)
    c = Cache(rng, [900, 2600], 1, 2, 64, False)
    s = Step(rng, c, 4, [5, 3], scale=1.0)
    got = torch.empty((8, 4, 64), device="cuda")
    assert s.step.plan_trees(i32(s.cu), s.parent, s.status) == sonic.OK
    for scale in (0.01, 4.0):
        ws = torch.empty(sonic.tree_decode_workspace_bytes(2, s.step.max_nodes, 4, 64, 2600), dtype=torch.uint8, device="cuda")
        dev = c.dev
        assert sonic.tree_decode(s.step.plan, dev.k, dev.v, dev.row_off, dev.length, *(bf16_to_device(x) for x in (s.q, s.k, s.v)), got, ws,
                                 s.status, s.step.max_nodes, 2600, softmax_scale=scale) == sonic.OK
        for b in range(2):
            o, n, a, e = int(c.off[b]), int(c.lens[b]), s.cu[b], s.cu[b + 1]
            want = OT.attend(bf16_bits_to_f64(s.q[a:e]), c.values[0][o:o + n], c.values[1][o:o + n], bf16_bits_to_f64(s.k[a:e]),
                             bf16_bits_to_f64(s.v[a:e]), s.parents[b], scale=scale)
            # a score is the sum of 64 products, off by 64 * 2^-24 of their magnitudes' sum at most, and so its exponential
            size = scale * 64 * np.abs(bf16_bits_to_f64(s.q[a:e])).max() * np.abs(c.values[0][o:o + n]).max()
            bar = 2 * (EPS + 64 * size * 2.0 ** -24) * max(np.abs(c.values[1][o:o + n]).max(), np.abs(bf16_bits_to_f64(s.v[a:e])).max())
            assert np.abs(got[a:e].double().cpu().numpy() - want).max() <= bar


# ------------------------------------------------------------------ values that are no numbers
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("out", ["fp32", "bf16"])
def test_a_nodes_values_reach_only_the_nodes_that_see_it(value, q4, out):
    H.need_gpu()
    rng = np.random.default_rng(31)
    for lens, nodes in (([40, 3], [20, 40]), ([1500, 0], [50, 6])):
        c = Cache(rng, lens, 1, 2, 128, q4)
        s = Step(rng, c, 6, nodes)
        bits = W.f32_to_bf16_bits(np.array([value], np.float32))[0]
        s.v[4, 1, 70] = bits                                     # node 4 of request 0
        s.v[int(s.cu[1]) + 5, 0, 3] = bits                       # node 5 of request 1
        s.k[3, 0, 5] = W.f32_to_bf16_bits(np.array([np.nan], np.float32))[0]
        got = s.run(out)
        for b in range(2):
            want, _ = s.expect(b)
            mine = got[s.cu[b]:s.cu[b + 1]]
            assert np.array_equal(np.isnan(mine), np.isnan(want)) and np.array_equal(np.isinf(mine), np.isinf(want))
            fine = np.isfinite(want)
            assert 0 < fine.sum() < want.size
            assert np.array_equal(mine[np.isinf(want)], want[np.isinf(want)])
            top = max(np.abs(x[np.isfinite(x)]).max() for x in (c.values[1], bf16_bits_to_f64(s.v)))
            assert np.abs(mine[fine] - want[fine]).max() <= BAR[out] * top


@pytest.mark.parametrize("where", [0, 17, 999])
def test_infinite_values_of_the_cache(where):
    """Seen by every node: an infinite output, NaN where both signs meet; the cache's last row is loaded more than once."""
    H.need_gpu()
    rng = np.random.default_rng(33)
    c = Cache(rng, [1000, 7], 1, 2, 64, False)
    o = int(c.off[0])
    for row, at, bits in ((where, 5, 0x7F80), (where, 9, 0xFF80), (where, 11, 0x7F80), ((where + 400) % 1000, 11, 0xFF80), (where, 20, 0x7FC0)):
        c.bits[1][o + row, 1, at] = bits
    c.dev.v.copy_(bf16_to_device(c.bits[1]))
    c.values[1] = bf16_bits_to_f64(c.bits[1])
    s = Step(rng, c, 4, [9, 4])
    for out in ("fp32", "bf16"):
        got = s.run(out)[:9]
        want, top = s.expect(0)
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and np.array_equal(np.isnan(got), np.isnan(want))
        fine = np.isfinite(want)
        assert np.abs(got[fine] - want[fine]).max() <= BAR[out] * top


# ------------------------------------------------------------------ errors
@pytest.mark.parametrize("cu,parent,nodes", [([0, 3, 2], [-1, 0, 0, 0], 4), ([1, 2, 4], [-1] * 4, 4), ([0, 2, 5], [-1] * 4, 4),
                                             ([0, 3, 4], [-1] * 4, 2), ([0, 2, 4], [-1, 1, -1, 0], 4), ([0, 2, 4], [-1, 0, -2, 0], 4),
                                             ([0, 2, 4], [-1, 0, -1, 7], 4)])
def test_malformed_trees(cu, parent, nodes):
    """The plan raises, and nothing is written behind it."""
    H.need_gpu()
    rng = np.random.default_rng(3)
    c = Cache(rng, [30, 300], 1, 2, 64, False)
    step = DraftStep(2, 4, nodes)
    assert step.plan_trees(i32(cu), i32(parent), c.status) == sonic.OK
    assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
    out = torch.full((4, 4, 64), 7.0, device="cuda")
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert c.dev.tree_decode(step.plan, q, x, x, out, c.status, nodes, 300) == sonic.OK
    assert torch.all(out == 7.0) and int(c.status.item()) == sonic.ERR_BAD_LAYOUT
    # the request at fault has no nodes, whatever is done about the status word
    c.status.zero_()
    assert c.dev.tree_decode(step.plan, q, x, x, out, c.status, nodes, 300) == sonic.OK
    torch.cuda.synchronize()


@pytest.mark.parametrize("bound", [300, 5000])
def test_lengths_past_the_bound_and_pending_errors(bound):
    H.need_gpu()
    rng = np.random.default_rng(4)
    c = Cache(rng, [30, 300, 50], 1, 2, 64, False)
    s = Step(rng, c, 4, [3, 4, 5])
    for length in (-1, bound + 1):
        c.dev.length.copy_(i32([30, length, 50]))
        got = s.run(max_ctx=bound)
        assert int(s.status.item()) == sonic.ERR_CAPACITY
        assert np.all(got[3:7] == 7.0)
        s.check(got, skip=(1,))
        c.dev.length.copy_(i32(c.lens))
        s.check(s.run(max_ctx=bound), skip=(None,))      # a capacity error that is pending stops nothing
        s.status.zero_()
    for code in (sonic.ERR_BAD_LAYOUT, sonic.ERR_INVALID_ARG):
        s.status.fill_(code)
        assert np.all(s.run(max_ctx=bound) == 7.0) and int(s.status.item()) == code
        s.status.zero_()


def test_a_plan_that_was_never_made_reads_nothing_outside():
    """Zeros, and a plan of many more nodes: no nodes, or none outside of the call's rows."""
    H.need_gpu()
    rng = np.random.default_rng(6)
    c = Cache(rng, [30, 300], 1, 2, 64, False)
    s = Step(rng, c, 4, [3, 4])
    assert np.all(s.run(plan=False) == 7.0)
    big = DraftStep(2, 400, 200)
    assert big.plan_trees(i32([0, 200, 400]), None, s.status) == sonic.OK
    s.step.plan.copy_(big.plan[:s.step.plan.numel()])
    assert np.all(s.run(plan=False) == 7.0)
    s.check(s.run())


# ------------------------------------------------------------------ how it is called
def test_one_workspace_for_calls_of_other_shapes():
    H.need_gpu()
    rng = np.random.default_rng(8)
    shapes = [([3000, 40], 4, 2, 64, [9, 3]), ([500] * 5, 8, 8, 128, [4] * 5), ([9000], 8, 1, 64, [70]), ([20], 2, 2, 64, [1])]
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")     # not zeros
    for lens, Hq, Hkv, d, nodes in shapes + shapes[::-1]:
        for q4 in (False, True):
            s = Step(rng, Cache(rng, lens, 1, Hkv, d, q4), Hq, nodes)
            s.c.dev.workspaces.made["tree"] = [ws]
            s.check(s.run())


def test_captured_steps_on_two_streams():
    """Two graphs with workspaces of their own, replayed side by side after the lengths, the trees and the inputs changed, with
    eager work between the replays."""
    H.need_gpu()
    rng = np.random.default_rng(12)
    made = []
    for q4 in (False, True):
        c = Cache(rng, [900, 2000, 33], 1, 2, 128, q4)
        s = Step(rng, c, 8, [12, 7, 5], spare=6)
        stream = torch.cuda.Stream()
        dev = [bf16_to_device(x) for x in (s.q, s.k, s.v)]
        cu, parent, out = i32(s.cu), s.parent.clone(), torch.zeros((s.N, 8, 128), device="cuda")

        def call():
            assert s.step.plan_trees(cu, parent, s.status) == sonic.OK
            assert c.dev.tree_decode(s.step.plan, *dev, out, s.status, s.step.max_nodes, 2000) == sonic.OK
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        made.append((c, s, stream, dev, cu, parent, out, graph))
    for lens, nodes in (([900, 2000, 33], [12, 7, 5]), ([5, 0, 33], [2, 12, 12]), ([899, 700, 32], [0, 1, 9])):
        for c, s, stream, dev, cu, parent, out, graph in made:
            c.lens[:] = lens
            c.dev.length.copy_(i32(c.lens))
            s.nodes, s.parents = nodes, [tree(rng, n) for n in nodes]
            s.cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
            s.q = normal_bits(rng, s.N, 8, 128)
            dev[0].copy_(bf16_to_device(s.q))
            cu.copy_(i32(s.cu))
            parent[:s.cu[-1]] = i32(np.concatenate(s.parents))
            out.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(2):
            for c, s, stream, *_, graph in made:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for c, s, stream, dev, cu, parent, out, graph in made:
            s.check(out.double().cpu().numpy())


def test_a_stream_of_its_own_and_the_same_result_again():
    H.need_gpu()
    rng = np.random.default_rng(13)
    s = Step(rng, Cache(rng, [4000, 100], 1, 2, 128, False), 8, [30, 4])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    first = s.run(stream=stream)
    s.check(first)
    for _ in range(3):
        assert np.array_equal(first, s.run())


def test_rows_past_4_gib():
    """A request whose rows start, and end, more than 4 GiB into the cache."""
    H.need_gpu()
    rng = np.random.default_rng(14)
    Hkv, d, rows = 16, 128, 1_400_000                         # 4 KiB a row and tensor: 5.7 GB each
    k, v = (torch.zeros((rows, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n, last = 300, 1_399_700
    bits = [normal_bits(rng, n, Hkv, d) for _ in range(2)]
    for x, y in zip((k, v), bits):
        x[last:] = bf16_to_device(y)
    step = DraftStep(2, 6, 4)
    status = i32([0])
    cu, parent = [0, 4, 6], [-1, 0, 1, 1, -1, 0]
    assert step.plan_trees(i32(cu), i32(parent), status) == sonic.OK
    q, kn, vn = normal_bits(rng, 6, Hkv, d), normal_bits(rng, 6, Hkv, d), normal_bits(rng, 6, Hkv, d)
    # the second request has zeros before its rows: their scores are zero, their values count for nothing
    length = [n, 1_400_000]
    out = torch.empty((6, Hkv, d), device="cuda")
    ws = torch.empty(sonic.tree_decode_workspace_bytes(2, 4, Hkv, d, rows), dtype=torch.uint8, device="cuda")
    assert sonic.tree_decode(step.plan, k, v, torch.tensor([last, 0], device="cuda"), i32(length), *(bf16_to_device(x) for x in (q, kn, vn)), out,
                             ws, status, 4, rows) == sonic.OK
    assert int(status.item()) == 0
    bar = 2 * (EPS + 1024 * 2.0 ** -24)       # a lane adds up to some 700 blocks' sums, one after the other
    f = [bf16_bits_to_f64(x) for x in (q, kn, vn, *bits)]
    want = OT.attend(f[0][:4], f[3], f[4], f[1][:4], f[2][:4], parent[:4])
    assert np.abs(out[:4].double().cpu().numpy() - want).max() <= bar * np.abs(f[4]).max()
    for i in range(2):
        for h in range(Hkv):
            kk, vv = (np.concatenate([f[a][:, h], f[a - 2][4:5 + i, h]]) for a in (3, 4))
            s = kk @ f[0][4 + i, h] / np.sqrt(d)
            top = max(s.max(), 0.0)
            p = np.exp(s - top)
            want = (p @ vv) / (p.sum() + last * np.exp(-top))
            assert np.abs(out[4 + i, h].double().cpu().numpy() - want).max() <= bar * np.abs(vv).max()


# ------------------------------------------------------------------ how a call is cut
@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [17, 33])
def test_every_cut(B, d, q4, out):
    """Tiles of 16 to 128 rows in four and eight waves: 136 and 264 (request, kv-head) pairs, up to 16, 32, 64, 128 and 136 rows a
    kv-head, one long context among short ones; each with all values numbers, and with some that are none."""
    H.need_gpu()
    rng = np.random.default_rng(B + d + q4)
    lens = rng.integers(0, 60, B)
    lens[3] = 3300
    c = Cache(rng, lens, 1, 8, d, q4)
    for most in (8, 16, 32, 64, 68):
        nodes = [int(x) for x in rng.integers(0, 4, B)]
        nodes[3], nodes[5] = most // 2 + 1, most
        s = Step(rng, c, 16, nodes)
        s.check(s.run(out), out)
        s.v[int(s.cu[5]) + 2, 4, 9] = 0x7FC0                       # one node's value: NaN
        got = s.run(out)
        for b in (3, 5):
            want, top = s.expect(b)
            mine = got[s.cu[b]:s.cu[b + 1]]
            assert np.array_equal(np.isnan(mine), np.isnan(want)), b
            fine = ~np.isnan(want)
            assert np.all(np.abs(mine[fine] - want[fine]) <= BAR[out] * top)


def test_two_calls_at_once():
    """Side by side on two streams, each with its own workspace and the same cache and plan."""
    H.need_gpu()
    rng = np.random.default_rng(41)
    c = Cache(rng, [6000, 300], 1, 2, 128, False)
    steps = [Step(rng, c, 8, [9, 3]) for _ in range(2)]
    steps[1].parents, steps[1].parent = steps[0].parents, steps[0].parent
    streams = [torch.cuda.Stream() for _ in range(2)]
    assert steps[0].step.plan_trees(i32(steps[0].cu), steps[0].parent, c.status) == sonic.OK
    dev = [[bf16_to_device(x) for x in (s.q, s.k, s.v)] for s in steps]
    out = [torch.zeros((12, 8, 128), device="cuda") for _ in steps]
    ws = [torch.empty(sonic.tree_decode_workspace_bytes(2, 9, 8, 128, 6000), dtype=torch.uint8, device="cuda") for _ in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, stream in enumerate(streams):
            assert sonic.tree_decode(steps[0].step.plan, c.dev.k, c.dev.v, c.dev.row_off, c.dev.length, *dev[i], out[i], ws[i], c.status, 9, 6000,
                                     stream=stream) == sonic.OK
    torch.cuda.synchronize()
    for s, o in zip(steps, out):
        s.check(o.double().cpu().numpy())
