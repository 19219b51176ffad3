"""The end of a step over drafted tokens (the confirmed path, its rows in the cache, its tokens in the history) against the
oracle, exactly; and whole steps, as a program makes them, against token by token decode."""
import numpy as np
import pytest
import torch

from oracle import q4 as OQ
from oracle import tree as OT
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import CompactCache, DraftStep, Q4Cache, bf16_to_device, bf16_to_host
from tests import gpu_helpers as H
from tests.test_gpu_q4 import EPS, Cache, i32, normal_bits
from tests.test_gpu_tree import BAR, tree

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ the confirmed path
class Accept:
    def __init__(self, rng, nodes, kind="bushy", spare=2, tokens=4):
        self.nodes, self.parents = nodes, [tree(rng, n, kind) for n in nodes]
        self.cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        self.N, B = int(self.cu[-1]) + spare, len(nodes)
        self.token = rng.integers(0, tokens, self.N).astype(np.int32)
        self.chosen = rng.integers(0, tokens, self.N).astype(np.int32)
        self.parent = None if kind == "chain" else i32(np.concatenate(self.parents + [np.zeros(spare, int)]))
        self.status = i32([0])
        self.step = DraftStep(B, self.N, max(max(nodes), 1))
        assert self.step.plan_trees(i32(self.cu), self.parent, self.status) == sonic.OK
        self.step.path.fill_(-9)
        self.hist_len = rng.integers(0, 9, B).astype(np.int32)
        self.hist_cap = self.hist_len + np.array(nodes) + 1
        self.hist_off = np.concatenate([[0], np.cumsum(self.hist_cap)])[:-1].astype(np.int64)
        self.tokens = rng.integers(100, 200, int(self.hist_cap.sum())).astype(np.int32)

    def run(self, history=True):
        kw = {}
        self.dev_len, self.dev_tokens = i32(self.hist_len), i32(self.tokens)
        if history:
            kw = dict(tokens=self.dev_tokens, token_off=torch.tensor(self.hist_off, device="cuda"), token_cap=i32(self.hist_cap),
                      token_len=self.dev_len)
        assert self.step.accept(self.parent, i32(self.token), self.status, chosen=i32(self.chosen), **kw) == sonic.OK
        torch.cuda.synchronize()
        return self

    def check(self, history=True, full=()):
        path, path_len, after = (x.cpu().numpy() for x in (self.step.path, self.step.path_len, self.step.next_token))
        tokens, lens = self.tokens.copy(), self.hist_len.copy()
        for b, n in enumerate(self.nodes):
            s, e = self.cu[b], self.cu[b + 1]
            want, token = OT.accepted(self.parents[b].tolist(), self.token[s:e], self.chosen[s:e])
            if b in full:
                want, token = [], -1
            assert path[s:e].tolist() == want + [-1] * (n - len(want)), b
            assert (path_len[b], after[b]) == (len(want), token)
            if history:
                o = int(self.hist_off[b] + lens[b])
                tokens[o:o + len(want)] = self.token[s:e][want]
                lens[b] += len(want)
        assert np.all(path[self.cu[-1]:] == -9)
        assert np.array_equal(self.dev_tokens.cpu().numpy(), tokens) and np.array_equal(self.dev_len.cpu().numpy(), lens)


@pytest.mark.parametrize("kind", ["bushy", "chain", "star", "forest"])
@pytest.mark.parametrize("nodes", [[1], [0], [7, 0, 64, 65, 1], [256, 200, 129, 128, 127, 63], [5] * 300])
def test_paths(nodes, kind):
    H.need_gpu()
    for tokens in (1, 2, 4, 1000):
        rng = np.random.default_rng(len(nodes) + tokens)
        Accept(rng, nodes, kind, tokens=tokens).run().check()
    Accept(np.random.default_rng(3), nodes, kind).run(history=False).check(history=False)


def test_a_whole_chain_confirmed():
    H.need_gpu()
    a = Accept(np.random.default_rng(1), [256, 3], "chain", tokens=1).run()
    a.check()
    assert a.step.path_len.tolist() == [256, 3]


def test_full_histories_and_pending_errors():
    H.need_gpu()
    a = Accept(np.random.default_rng(2), [6, 9, 4, 5], "chain", tokens=1)
    a.hist_cap[1] = a.hist_len[1] + 8          # one place short
    a.hist_len[2] = -1
    a.hist_cap[3] = -2 ** 31
    a.run().check(full=(1, 2, 3))
    assert int(a.status.item()) == sonic.ERR_CAPACITY
    a.run().check(full=(1, 2, 3))              # pending: stops nothing
    before = a.step.path.clone()
    a.status.fill_(sonic.ERR_BAD_LAYOUT)
    a.chosen[:] = -1
    a.run()
    assert torch.equal(before, a.step.path) and np.array_equal(a.dev_len.cpu().numpy(), a.hist_len)


# ------------------------------------------------------------------ rows to the end of a cache
def rows_of(c):
    """The cache's arrays on the host."""
    if c.q4:
        return [x.cpu().numpy().copy() for x in (c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale)]
    return [bf16_to_host(x).copy() for x in (c.dev.k, c.dev.v)]


def put(c, rows, at, bits):
    """Row `at` of the host arrays takes k and v."""
    for i, x in enumerate(bits):
        if c.q4:
            codes, scales = OQ.encode(x)
            rows[i][at], rows[2 + i][at] = OQ.pack(codes), scales
        else:
            rows[i][at] = x


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("Hkv,d", [(1, 64), (2, 128), (8, 128), (5, 64)])
def test_append(Hkv, d, q4):
    H.need_gpu()
    rng = np.random.default_rng(Hkv + q4)
    for counts in ([3, 0, 7, 1], [40, 1, 0, 300], [1] * 70):
        B = len(counts)
        c = Cache(rng, rng.integers(0, 50, B), max(counts) + 2, Hkv, d, q4)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        n = int(cu[-1])
        bits = [normal_bits(rng, n + 1, Hkv, d) for _ in range(2)]
        for select in (False, True):
            rows = rows_of(c)
            kw, take = {}, [list(range(m)) for m in counts]
            if select:
                take = [list(rng.integers(0, m, rng.integers(0, m + 1))) if m else [] for m in counts]     # any order, repeats
                flat = np.full(n + 1, -5)
                for s, t in zip(cu, take):
                    flat[s:s + len(t)] = t
                kw = dict(select=i32(flat), select_len=i32([len(t) for t in take]))
                c.dev.length.copy_(i32(c.lens))
            assert c.dev.append(i32(cu), *(bf16_to_device(x) for x in bits), c.status, max(counts), **kw) == sonic.OK
            torch.cuda.synchronize()
            assert int(c.status.item()) == 0
            for b, t in enumerate(take):
                for j, x in enumerate(t):
                    put(c, rows, int(c.off[b] + c.lens[b]) + j, [y[cu[b] + x] for y in bits])
            assert all(np.array_equal(x, y) for x, y in zip(rows_of(c), rows))
            assert c.dev.length.tolist() == [int(m) + len(t) for m, t in zip(c.lens, take)]


@pytest.mark.parametrize("q4", [False, True])
def test_append_errors_leave_the_request_and_do_the_others(q4):
    H.need_gpu()
    rng = np.random.default_rng(5)
    B, m = 40, 3
    cu = (np.arange(B + 1) * m).astype(np.int32)
    bits = [normal_bits(rng, B * m, 2, 64) for _ in range(2)]
    full = np.tile(np.arange(m), B)

    def case(code, cu=cu, select=full, count=None, cap=None, length=None, max_rows=m, bad=(7,)):
        c = Cache(rng, [10] * B, m, 2, 64, q4)
        count = np.full(B, m) if count is None else count
        for name, x in (("row_cap", cap), ("length", length)):
            if x is not None:
                getattr(c.dev, name)[7] = x
        before, rows = c.dev.length.tolist(), rows_of(c)
        for _ in range(1):
            assert c.dev.append(i32(cu), *(bf16_to_device(x) for x in bits), c.status, max_rows, select=i32(select),
                                select_len=i32(count)) == sonic.OK
        assert int(c.status.item()) == code
        for b in range(B):
            if b not in bad:
                for j in range(m):
                    put(c, rows, int(c.off[b]) + 10 + j, [x[b * m + j] for x in bits])
        assert all(np.array_equal(x, y) for x, y in zip(rows_of(c), rows))
        assert c.dev.length.tolist() == [n if b in bad else n + m for b, n in enumerate(before)]

    at = lambda a, i, x: np.concatenate([a[:i], [x], a[i + 1:]])  # noqa: E731
    case(sonic.ERR_CAPACITY, cap=12)
    case(sonic.ERR_CAPACITY, cap=-5)
    case(sonic.ERR_CAPACITY, cap=-2 ** 31)
    case(sonic.ERR_BAD_LAYOUT, length=-1)
    case(sonic.ERR_BAD_LAYOUT, select=at(full, 22, 3))
    case(sonic.ERR_BAD_LAYOUT, select=at(full, 23, -1))
    case(sonic.ERR_BAD_LAYOUT, count=at(np.full(B, m), 7, m + 1))
    case(sonic.ERR_BAD_LAYOUT, count=at(np.full(B, m), 7, -1))
    case(sonic.ERR_BAD_LAYOUT, cu=at(cu, B, B * m + 1), bad=(B - 1,))
    case(sonic.ERR_INVALID_ARG, max_rows=m - 1, bad=range(B))


def test_append_and_pending_errors():
    H.need_gpu()
    rng = np.random.default_rng(6)
    c = Cache(rng, [4, 5], 6, 2, 64, False)
    x = bf16_to_device(normal_bits(rng, 4, 2, 64))
    for code, moves in ((sonic.ERR_CAPACITY, True), (sonic.ERR_BAD_LAYOUT, False)):
        c.status.fill_(code)
        before, rows = c.dev.length.clone(), rows_of(c)
        assert c.dev.append(i32([0, 2, 4]), x, x, c.status, 2) == sonic.OK
        assert torch.equal(c.dev.length, before + 2 if moves else before)
        assert moves or all(np.array_equal(a, b) for a, b in zip(rows, rows_of(c)))
    none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    c.status.zero_()
    before = c.dev.length.clone()
    assert c.dev.append(i32([0, 0, 0]), none, none, c.status, 0) == sonic.OK
    assert torch.equal(c.dev.length, before) and int(c.status.item()) == 0


def test_append_past_4_gib():
    H.need_gpu()
    rng = np.random.default_rng(7)
    rows, Hkv, d = 1_100_000, 16, 128
    c = CompactCache(rows, Hkv, d, [0, 1_099_990], [1_099_990, 10], "cuda", fill_bits=0)
    c.length.copy_(i32([1_099_980, 2]))
    bits = [normal_bits(rng, 7, Hkv, d) for _ in range(2)]
    status = i32([0])
    assert c.append(i32([0, 4, 7]), *(bf16_to_device(x) for x in bits), status, 4) == sonic.OK
    assert int(status.item()) == 0 and c.length.tolist() == [1_099_984, 5]
    for x, y in zip((c.k, c.v), bits):
        got = bf16_to_host(x[1_099_975:])
        want = np.zeros_like(got)
        want[5:9], want[17:20] = y[:4], y[4:]
        assert np.array_equal(got, want)
        assert not torch.any(x[:1_099_975])


# ------------------------------------------------------------------ whole steps
class Model:
    """A little model of two layers over a vocabulary of 50 tokens, the same for drafted and for generated tokens: a token's
    q, k and v of a layer are fixed, and its logits come from its last layer's output.  Plain torch, in 64 bits, so that a
    token's logits do not depend on how many are taken at once."""

    def __init__(self, rng, Hq, Hkv, d, V=50):
        self.q, self.k, self.v = (bf16_to_device(normal_bits(rng, 2, V, h, d)) for h in (Hq, Hkv, Hkv))
        self.out = torch.from_numpy(rng.standard_normal((2, Hq * d, V))).cuda()

    def logits(self, outs):
        return sum(torch.mm(o.double().reshape(o.shape[0], -1), w) for o, w in zip(outs, self.out)).float()


def make_caches(rng, lens, room, Hkv, d, q4):
    cap = np.array(lens) + room
    off = np.concatenate([[0], np.cumsum(cap)])[:-1].astype(np.int64)
    return [(Q4Cache if q4 else CompactCache)(int(cap.sum()), Hkv, d, off, cap, "cuda") for _ in range(2)]


@pytest.mark.parametrize("q4", [False, True])
def test_steps_generate_what_token_by_token_decode_does(q4):
    """Prompts through chains in two pieces; then steps over drafted trees, which contain the right continuation and wrong ones,
    with penalties and masks: the same tokens and caches as decode of one token at a time (fp32 outputs)."""
    H.need_gpu()
    rng = np.random.default_rng(21 + q4)
    B, Hq, Hkv, d, V, room = 3, 4, 2, 64, 50, 40
    prompts = [rng.integers(0, V, n) for n in (70, 9, 200)]
    model = Model(rng, Hq, Hkv, d, V)
    status = i32([0])
    rep, pres, freq = (torch.tensor(x, dtype=torch.float32, device="cuda") for x in ([1.3, 1.0, 1.1], [0.5, 0.0, 0.2], [0.1, 0.3, 0.0]))
    allowed = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (1, 2)).astype(np.int32)).cuda()

    def prompt_through(caches):
        """Both pieces of the prompts, chains of up to 256 nodes."""
        for part in (lambda p: p[:len(p) // 3], lambda p: p[len(p) // 3:]):
            pieces = [part(p) for p in prompts]
            cu = np.concatenate([[0], np.cumsum([len(p) for p in pieces])])
            t = torch.from_numpy(np.concatenate(pieces)).cuda()
            step = DraftStep(B, int(cu[-1]), 256)
            assert step.plan_trees(i32(cu), None, status) == sonic.OK
            for i, c in enumerate(caches):
                out = torch.empty((int(cu[-1]), Hq, d), device="cuda")
                assert c.tree_decode(step.plan, model.q[i][t], model.k[i][t], model.v[i][t], out, status, 256, 200) == sonic.OK
                assert c.append(i32(cu), model.k[i][t], model.v[i][t], status, 256) == sonic.OK

    def history():
        off = torch.tensor([0, 400, 800], device="cuda")
        tokens = torch.zeros(1200, dtype=torch.int32, device="cuda")
        for b, p in enumerate(prompts):
            tokens[400 * b:400 * b + len(p)] = i32(p)
        lens = i32([len(p) for p in prompts])
        return dict(tokens=tokens, token_off=off, token_len=lens), dict(prompt_len=lens.clone(), repetition=rep, presence=pres, frequency=freq)

    # token by token
    one = make_caches(rng, [len(p) for p in prompts], room, Hkv, d, q4)
    prompt_through(one)
    hist, how = history()
    now = i32([1, 2, 3])
    ws = torch.zeros(sonic.logits_process_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    said = []
    for _ in range(24):
        outs = []
        for i, c in enumerate(one):
            out = torch.empty((B, Hq, d), device="cuda")
            args = (model.q[i][now.long()], model.k[i][now.long()], model.v[i][now.long()], out, status, 250)
            assert (c.decode(*args) if q4 else c.decode_weighted(*args)) == sonic.OK
            outs.append(out)
        said.append(now.tolist())
        best = i32([0] * B)
        assert sonic.logits_process(model.logits(outs), best, ws, status, node_token=now, allowed=allowed.expand(B, 2).contiguous(),
                                    **hist, **how) == sonic.OK
        hist["tokens"][hist["token_off"] + hist["token_len"]] = now
        hist["token_len"] += 1
        now = best
    assert int(status.item()) == 0
    said = np.array(said)                                       # [24, B]

    # steps over trees of what was said, of wrong branches, and of branches that go wrong
    caches = make_caches(rng, [len(p) for p in prompts], room, Hkv, d, q4)
    prompt_through(caches)
    hist, how = history()
    done, now, steps = np.zeros(B, int), i32([1, 2, 3]), 0
    step = DraftStep(B, 40, 12)
    while done.min() < 23:
        parents, tokens = [], []
        for b in range(B):
            ahead, first = said[done[b] + 1:done[b] + 1 + rng.integers(0, 5), b], int(now[b])
            parent, token, last = [-1], [first], 0
            for right in ahead:
                pair = [int(right), int(right + 1) % V]
                if rng.random() < 0.5:
                    pair.reverse()
                parent += [last, last]
                token += pair
                last = len(token) - 2 + pair.index(int(right))
            parents.append(parent)
            tokens.append(token)
        cu = np.concatenate([[0], np.cumsum([len(p) for p in parents])])
        n = int(cu[-1])
        flat = lambda x: i32(np.concatenate([np.concatenate(x), np.zeros(40 - n, int)]))  # noqa: E731
        parent, token = flat(parents), flat(tokens)
        assert step.plan_trees(i32(cu), parent, status) == sonic.OK
        outs, rows = [], []
        for i, c in enumerate(caches):
            out = torch.zeros((40, Hq, d), device="cuda")
            k, v = model.k[i][token.long()], model.v[i][token.long()]
            assert c.tree_decode(step.plan, model.q[i][token.long()], k, v, out, status, 12, 250) == sonic.OK
            outs.append(out)
            rows.append((k, v))
        assert step.logits(model.logits(outs), status, node_token=token, allowed=allowed.expand(40, 2).contiguous(), **hist, **how) == sonic.OK
        assert step.accept(parent, token, status, **hist, token_cap=i32([400] * B)) == sonic.OK
        for c, (k, v) in zip(caches, rows):
            assert c.append(i32(cu), k, v, status, 12, select=step.path, select_len=step.path_len) == sonic.OK
        assert int(status.item()) == 0
        for b, m in enumerate(step.path_len.tolist()):
            assert m >= 1 and (m > 1 or len(parents[b]) == 1 or done[b] + 1 >= 24)
        done += np.array(step.path_len.tolist())
        now, steps = step.next_token.clone(), steps + 1
        for b in range(B):
            if done[b] < 24:
                assert int(now[b]) == said[done[b], b]
    assert steps < 20
    for b, p in enumerate(prompts):
        got = hist["tokens"][400 * b + len(p):400 * b + len(p) + 23].tolist()
        assert got == said[:23, b].tolist()
        m = len(p) + 23
        for c, o in zip(caches, one):
            rows = slice(int(c.row_off_host[b]), int(c.row_off_host[b]) + m)
            assert torch.equal(c.k[rows], o.k[rows]) and torch.equal(c.v[rows], o.v[rows])


def test_a_captured_step_replayed():
    """Plan, two layers, logits, accept and append as one graph, replayed step after step with the program's own work between:
    the caches, histories and tokens are those of the same calls made one by one."""
    H.need_gpu()
    B, Hq, Hkv, d, V, n = 2, 4, 2, 64, 50, 12
    runs = []
    for captured in (False, True):
        rng = np.random.default_rng(31)
        model = Model(rng, Hq, Hkv, d, V)
        caches = make_caches(rng, [60, 300], 40, Hkv, d, False)
        for c in caches:
            for x in (c.k, c.v):
                x.copy_(bf16_to_device(normal_bits(rng, x.shape[0], Hkv, d)))
            c.length.copy_(i32([60, 300]))
        status, step = i32([0]), DraftStep(B, n, 8)
        cu, parent, token, chosen = i32([0, 0, 0]), i32([0] * n), i32([0] * n), i32([0] * n)
        tokens, off, lens = i32(rng.integers(0, V, 200)), torch.tensor([0, 100], device="cuda"), i32([20, 30])
        out = [torch.zeros((n, Hq, d), device="cuda") for _ in caches]
        logits = torch.zeros((n, V), device="cuda")

        def attention():
            assert step.plan_trees(cu, parent, status) == sonic.OK
            for i, c in enumerate(caches):
                assert c.tree_decode(step.plan, q[i], k[i], v[i], out[i], status, 8, 340) == sonic.OK

        def rest():
            assert step.logits(logits, status, node_token=token, tokens=tokens, token_off=off, token_len=lens,
                               frequency=frequency) == sonic.OK
            assert step.accept(parent, token, status, chosen=chosen, tokens=tokens, token_off=off, token_cap=cap, token_len=lens) == sonic.OK
            for i, c in enumerate(caches):
                assert c.append(cu, k[i], v[i], status, 8, select=step.path, select_len=step.path_len) == sonic.OK
        frequency, cap = torch.full((B,), 0.5, device="cuda"), i32([100] * B)
        q, k, v = ([torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda") for _ in caches] for h in (Hq, Hkv, Hkv))
        parts = [attention, rest]
        if captured:
            attention()                                    # (no nodes yet: nothing changes)
            rest()
            torch.cuda.synchronize()
            graphs = []
            for part in parts:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    part()
                graphs.append(g.replay)
            parts = graphs
        seen = []
        for turn in range(4):
            nodes = [int(x) for x in rng.integers(1, 6, B)]
            m = sum(nodes)
            flat = np.concatenate([tree(rng, x) for x in nodes])
            cu.copy_(i32(np.concatenate([[0], np.cumsum(nodes)])))
            parent[:m] = i32(flat)
            token[:m] = i32(rng.integers(0, 3, m))
            for i in range(2):
                for x, table in ((q, model.q), (k, model.k), (v, model.v)):
                    x[i].copy_(table[i][token.long()])
            parts[0]()
            logits.copy_(model.logits(out))
            chosen[:m] = i32(rng.integers(0, 3, m))
            parts[1]()
            torch.cuda.synchronize()
            assert int(status.item()) == 0
            seen += [x.clone() for x in (step.path[:m], step.path_len, step.next_token, step.best[:m], lens, tokens, *[c.length for c in caches])]
        for c in caches:
            for b in range(B):
                rows = slice(int(c.row_off_host[b]), int(c.row_off_host[b]) + int(c.length[b]))
                seen += [c.k[rows].clone(), c.v[rows].clone()]
        runs.append(seen)
    assert len(runs[0]) == len(runs[1]) and all(torch.equal(a, b) for a, b in zip(*runs))
    assert runs[0][-1].shape[0] >= 304                     # every step adds its tree's first node at least
