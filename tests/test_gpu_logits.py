"""Logits with penalties, biases and masks on the GPU against the oracle, bit for bit: every operation is one 32-bit
rounding on both sides."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import tree as OT
from oracle.attention import bf16_bits_to_f64
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import CompactCache, DraftStep
from tests import gpu_helpers as H
from tests.test_gpu_q4 import i32
from tests.test_gpu_tree import tree

pytestmark = pytest.mark.gpu

f32 = lambda a: torch.tensor(np.asarray(a, np.float32), device="cuda")  # noqa: E731


class Call:
    """One call's inputs on both sides; what is None is left out of it."""

    def __init__(self, rng, B, V, bf16=False, nodes=None, hist=40, biases=3, mask="half", parts=("history", "penalties", "path"), spare=0):
        self.B, self.V, self.nodes = B, V, nodes
        n = B if nodes is None else sum(nodes) + spare
        self.n, self.cu = n, np.concatenate([[0], np.cumsum(nodes if nodes is not None else [1] * B)]).astype(np.int32)
        self.parents = [np.array([-1])] * B if nodes is None else [tree(rng, m) for m in nodes]
        x = (rng.standard_normal((n, V)) * 3).astype(np.float32)
        self.x = bf16_bits_to_f64(W.f32_to_bf16_bits(x)).astype(np.float32) if bf16 else x
        self.dev_x = torch.from_numpy(self.x).cuda().to(torch.bfloat16 if bf16 else torch.float32)
        ids = lambda m: np.minimum((V * rng.random(m) ** 2).astype(np.int32), V - 1)  # noqa: E731
        self.len = rng.integers(0, hist + 1, B).astype(np.int32)
        self.off = np.concatenate([[0], np.cumsum(self.len + 2)])[:-1].astype(np.int64)
        self.tokens = ids(int((self.len + 2).sum()))
        self.tokens[rng.random(len(self.tokens)) < 0.05] = -1
        self.tokens[rng.random(len(self.tokens)) < 0.05] = V
        self.prompt = (self.len * rng.random(B)).astype(np.int32)
        self.node_token = ids(n)
        self.rep, self.pres, self.freq = 1 + rng.random(B), rng.random(B), rng.random(B) / 3
        count = rng.integers(0, biases + 1, B) if biases else np.zeros(B, int)
        self.bias_cu = np.concatenate([[0], np.cumsum(count)]).astype(np.int32)
        self.bias_token = np.concatenate([ids(int(count.sum())), [0]]).astype(np.int32)     # repeats among them
        self.bias_value = (rng.standard_normal(len(self.bias_token)) * 4).astype(np.float32)
        self.parts = set(parts) | ({"biases"} if biases else set())
        self.allowed = None if mask is None else rng.random((n, V)) < (0.5 if mask == "half" else 2 / V)
        self.status = i32([0])
        self.step = None if nodes is None else DraftStep(B, n, max(max(nodes), 1))
        if self.step is not None:
            flat = np.concatenate(self.parents + [np.zeros(spare, int)])
            assert self.step.plan_trees(i32(self.cu), i32(flat), self.status) == sonic.OK

    def run(self, out=True, stream=None, ws=None):
        n, V, kw = self.n, self.V, {}
        if "history" in self.parts:
            kw.update(tokens=i32(self.tokens), token_off=torch.tensor(self.off, device="cuda"), token_len=i32(self.len), prompt_len=i32(self.prompt))
        if "penalties" in self.parts:
            kw.update(repetition=f32(self.rep), presence=f32(self.pres), frequency=f32(self.freq))
        if "path" in self.parts:
            kw.update(node_token=i32(self.node_token))
        if "biases" in self.parts:
            kw.update(bias_cu=i32(self.bias_cu), bias_token=i32(self.bias_token), bias_value=f32(self.bias_value))
        if self.allowed is not None:
            words = np.zeros((n, (V + 31) // 32 * 32), np.uint8)
            words[:, :V] = self.allowed
            kw["allowed"] = torch.from_numpy(np.packbits(words, axis=1, bitorder="little").view(np.int32)).cuda()
        if self.step is not None:
            kw.update(plan=self.step.plan, batch=self.B, max_nodes=self.step.max_nodes)
        self.best, self.value = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), 7.0, device="cuda")
        self.out = torch.full((n, V), 7.0, device="cuda") if out else None
        if ws is None:
            ws = torch.full((sonic.logits_process_workspace_bytes(n, V),), 255, dtype=torch.uint8, device="cuda")
        st = sonic.logits_process(self.dev_x, self.best, ws, self.status, best_value=self.value, out=self.out, stream=stream, **kw)
        assert st == sonic.OK, sonic.status_string(st)
        torch.cuda.synchronize()
        return self

    def check(self, skip=()):
        best, value = self.best.cpu().numpy(), self.value.cpu().numpy()
        out = None if self.out is None else self.out.cpu().numpy()
        has = lambda name: name in self.parts  # noqa: E731
        for b in range(self.B):
            rows = range(self.cu[b], self.cu[b + 1])
            if b in skip:
                assert np.all(best[rows] == -7) and np.all(value[rows] == 7.0) and (out is None or np.all(out[rows] == 7.0))
                continue
            o, m, p = int(self.off[b]), int(self.len[b]), int(self.prompt[b])
            prompt, generated = (self.tokens[o:o + p], self.tokens[o + p:o + m]) if has("history") else ([], [])
            bias = [(int(t), v) for t, v in zip(self.bias_token[self.bias_cu[b]:self.bias_cu[b + 1]],
                                                self.bias_value[self.bias_cu[b]:self.bias_cu[b + 1]])] if has("biases") else []
            for i, row in enumerate(rows):
                path = self.node_token[self.cu[b] + np.array(OT.path_of(self.parents[b], i))] if has("path") else []
                rep, pres, freq = (self.rep[b], self.pres[b], self.freq[b]) if has("penalties") else (1, 0, 0)
                x, t, v = OT.logits_row(self.x[row], prompt, list(generated) + list(path), np.float32(rep), np.float32(pres), np.float32(freq),
                                        bias, None if self.allowed is None else self.allowed[row])
                assert (best[row], value[row]) == (t, v), (b, i)
                if out is not None:
                    assert np.array_equal(out[row], x, equal_nan=True), (b, i)
        rest = slice(int(self.cu[-1]), None)
        assert np.all(best[rest] == -7) and np.all(value[rest] == 7.0)


VOCABS = [1, 2, 31, 33, 257, 4095, 4096, 4097, 12289, 50257]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", VOCABS)
def test_rows_of_one_token_a_request(V, bf16):
    H.need_gpu()
    rng = np.random.default_rng(V + bf16)
    for B, mask in ((1, None), (5, "half"), (3, "few")):
        Call(rng, B, V, bf16, mask=mask).run().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", VOCABS)
def test_rows_of_trees(V, bf16):
    H.need_gpu()
    rng = np.random.default_rng(2 * V + bf16)
    Call(rng, 3, V, bf16, nodes=[5, 0, 9], spare=2).run().check()


def test_large_trees_and_long_histories():
    H.need_gpu()
    rng = np.random.default_rng(7)
    Call(rng, 2, 3001, nodes=[256, 40], hist=3000).run().check()
    Call(rng, 40, 9001, nodes=[3] * 40, hist=900, mask="few", biases=300).run(out=False).check()


@pytest.mark.parametrize("parts", [(), ("history",), ("penalties",), ("path",), ("history", "penalties"), ("path", "penalties")])
def test_what_a_program_leaves_out(parts):
    H.need_gpu()
    rng = np.random.default_rng(len(parts))
    for biases, mask in ((0, None), (2, None), (0, "half")):
        Call(rng, 4, 700, parts=parts, biases=biases, mask=mask).run().check()
        Call(rng, 2, 700, nodes=[3, 4], parts=parts, biases=biases, mask=mask).run().check()


def test_ties_infinities_and_nan():
    H.need_gpu()
    rng = np.random.default_rng(11)
    c = Call(rng, 6, 9001, parts=(), biases=0, mask=None)
    c.x[:] = np.round(c.x)
    c.x[0] = 2.0                                # all equal: token 0
    c.x[1, [8999, 5000, 300]] = 50.0            # equal in several pieces
    c.x[2] = -np.inf                            # nothing
    c.x[3] = np.nan
    c.x[4, 17], c.x[4, 4096], c.x[4, 9000] = np.nan, np.inf, np.inf
    c.x[5] = -np.inf
    c.x[5, 9000] = -3e38
    c.dev_x = torch.from_numpy(c.x).cuda()
    c.run().check()
    assert c.best.tolist()[:5] == [0, 300, -1, -1, 4096] and c.best.tolist()[5] == 9000


def test_a_mask_that_leaves_nothing():
    H.need_gpu()
    c = Call(np.random.default_rng(12), 3, 5000)
    c.allowed[1] = False
    c.run().check()
    assert int(c.best[1]) == -1 and float(c.value[1]) == -np.inf


def test_errors_leave_the_other_requests_to_be_done():
    H.need_gpu()
    for change in (lambda c: c.len.__setitem__(2, -1), lambda c: c.prompt.__setitem__(2, -1),
                   lambda c: c.prompt.__setitem__(2, c.len[2] + 1), lambda c: c.bias_cu.__setitem__(3, c.bias_cu[2] - 1)):
        for nodes in (None, [2, 3, 2, 1]):
            c = Call(np.random.default_rng(13), 4, 5000, nodes=nodes)
            cu = c.bias_cu.copy()
            change(c)
            skip = (2,) if np.array_equal(cu, c.bias_cu) else (2, 3)     # the next one's entries start elsewhere
            c.run()
            assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
            if skip == (2,):
                c.check(skip=skip)
    c = Call(np.random.default_rng(14), 4, 5000)
    c.status.fill_(sonic.ERR_CAPACITY)
    c.run().check()                                                       # stops nothing
    c.status.fill_(sonic.ERR_INVALID_ARG)
    c.run().check(skip=range(4))
    assert int(c.status.item()) == sonic.ERR_INVALID_ARG


def test_two_streams_and_graphs():
    H.need_gpu()
    rng = np.random.default_rng(15)
    calls = [Call(rng, 3, 20001, nodes=[4, 2, 9]), Call(rng, 5, 33333, True)]
    made = []
    for c in calls:
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            best, value, out = torch.zeros(c.n, dtype=torch.int32, device="cuda"), torch.zeros(c.n, device="cuda"), torch.zeros((c.n, c.V), device="cuda")
            ws = torch.zeros(sonic.logits_process_workspace_bytes(c.n, c.V), dtype=torch.uint8, device="cuda")
            kw = dict(plan=c.step.plan, batch=c.B, max_nodes=c.step.max_nodes) if c.step else {}
            token = i32(c.node_token)
            call = lambda: sonic.logits_process(c.dev_x, best, ws, c.status, node_token=token, repetition=rep, best_value=value, out=out, **kw)  # noqa: E731,B023
            rep = f32(c.rep)
            assert call() == sonic.OK
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            assert call() == sonic.OK
        made.append((c, stream, graph, best, value, out, token, rep, ws))
    for turn in range(3):
        for c, stream, graph, best, value, out, token, rep, ws in made:
            c.x = c.x[:, ::-1].copy()
            c.dev_x.copy_(torch.from_numpy(c.x))
            out.fill_(7.0)
        torch.cuda.synchronize()
        for c, stream, graph, *_ in made:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for c, stream, graph, best, value, out, *_ in made:
            c.best, c.value, c.out = best, value, out
            c.parts, c.allowed = {"path", "penalties"}, None
            c.pres, c.freq = np.zeros(c.B), np.zeros(c.B)
            c.check()


def test_elements_past_32_bits():
    """17,000 rows of 130,001 bf16 logits, 2.2e9 of them: the last rows as a call of their own does them."""
    H.need_gpu()
    n, V = 17000, 130001
    gen = torch.Generator(device="cuda").manual_seed(16)
    some = torch.randn((40, V), device="cuda", generator=gen).to(torch.bfloat16)
    x = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    x[:20], x[-20:] = some[:20], some[20:]
    best, value = [torch.zeros(m, dtype=torch.int32, device="cuda") for m in (n, 40)], [torch.zeros(m, device="cuda") for m in (n, 40)]
    token = torch.zeros(n, dtype=torch.int32, device="cuda")
    token[-20:] = some[20:].argmax(1).int()
    rep, status = torch.full((n,), 3.0, device="cuda"), i32([0])
    out = torch.zeros((40, V), device="cuda")
    for i, (rows, t, o) in enumerate(((x, token, None), (some, torch.cat([token[:20], token[-20:]]), out))):
        ws = torch.empty(sonic.logits_process_workspace_bytes(len(t), V), dtype=torch.uint8, device="cuda")
        assert sonic.logits_process(rows, best[i], ws, status, node_token=t, repetition=rep[:len(t)], best_value=value[i], out=o) == sonic.OK
    torch.cuda.synchronize()
    assert torch.equal(torch.cat([best[0][:20], best[0][-20:]]), best[1]) and torch.equal(torch.cat([value[0][:20], value[0][-20:]]), value[1])
    want = some.float().cpu().numpy()          # (on the host: a division of a GPU tensor by a number is a product with its inverse)
    at = (np.arange(40), np.concatenate([token[:20].cpu().numpy(), token[-20:].cpu().numpy()]))
    want[at] = np.where(want[at] > 0, want[at] / np.float32(3), want[at] * np.float32(3))
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(value[1].cpu().numpy(), want.max(1))


def test_many_biases_and_histories_without_a_prompt():
    """More biases than a workgroup has threads, a token several times among them; all of a history generated."""
    H.need_gpu()
    for nodes in (None, [3, 1]):
        c = Call(np.random.default_rng(17), 2, 700, nodes=nodes, hist=3000, biases=0)
        rng = np.random.default_rng(18)
        c.bias_cu = np.array([0, 1400, 2011], np.int32)
        c.bias_token = rng.integers(0, 700, 2011).astype(np.int32)
        c.bias_value = rng.standard_normal(2011).astype(np.float32)
        c.parts.add("biases")
        c.prompt[:] = 0
        c.run().check()
        c.prompt[:] = c.len
        c.run(out=False).check()


def test_histories_and_biases_without_an_entry():
    """Empty tensors, as a batch has them in which no request has any: as if they were left out."""
    H.need_gpu()
    c = Call(np.random.default_rng(19), 3, 500, hist=0, biases=0, parts=("penalties", "path"))
    c.run().check()
    want = c.out.clone()
    none, zeros = i32([]), i32([0, 0, 0])
    c.tokens, c.len, c.prompt = np.zeros(0, np.int32), np.zeros(3, np.int32), np.zeros(3, np.int32)
    c.bias_cu, c.bias_token, c.bias_value = np.zeros(4, np.int32), np.zeros(0, np.int32), np.zeros(0, np.float32)
    c.parts |= {"history", "biases"}
    c.run()
    assert torch.equal(c.out, want) and int(c.status.item()) == 0
    assert none.data_ptr() == 0 and zeros.data_ptr() != 0


def test_a_step_without_nodes():
    """Room for nodes but none, and no room at all: every call returns, nothing is written."""
    H.need_gpu()
    for n in (0, 4):
        status, step = i32([0]), DraftStep(2, n, 4)
        cu, tokens = i32([0, 0, 0]), i32([5] * n)
        x = torch.full((n, 100), 3.0, device="cuda")
        assert step.plan_trees(cu, tokens, status) == sonic.OK
        assert step.logits(x, status, node_token=tokens) == sonic.OK
        assert step.accept(tokens, tokens, status) == sonic.OK
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and step.path_len.tolist() == [0, 0] and step.next_token.tolist() == [-1, -1]
        assert torch.all(step.best == 0)
        c = CompactCache(8, 2, 64, [0, 4], [4, 4], "cuda")
        c.length.copy_(i32([3, 4]))
        k = torch.zeros((n, 2, 64), dtype=torch.bfloat16, device="cuda")
        q = torch.zeros((n, 4, 64), dtype=torch.bfloat16, device="cuda")
        out = torch.full((n, 4, 64), 7.0, device="cuda")
        assert c.tree_decode(step.plan, q, k, k, out, status, 4, 4) == sonic.OK
        assert c.append(cu, k, k, status, 4, select=step.path, select_len=step.path_len) == sonic.OK
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and c.length.tolist() == [3, 4] and torch.all(out == 7.0)
