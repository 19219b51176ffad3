"""Refusals of the entry points of a step over drafted tokens, and of their binding.  Nothing is enqueued in any of
these calls, so they run on the CPU, with pointers that nothing reads."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import tree as OT
from paper_2601_21927_amd import sonic

P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4098)   # 2-byte aligned only
BIG = 1 << 40


def call(name, names, values, **change):
    args = dict(zip(names.split(), values))
    assert set(change) <= set(args) and len(args) == len(values), change
    args.update(change)
    return getattr(sonic.lib(), name)(*args.values())


def plan(**c):
    return call("sonic_tree_plan", "B N nodes cu parent plan bytes status stream", [0, 8, 4, P, P, P, BIG, P, None], **c)


def decode(**c):
    return call("sonic_tree_decode", "B N nodes Hq Hkv d ctx plan bytes kc ks vc vs off len q kn vn scale out bf16 ws wbytes status stream",
                [0, 8, 4, 4, 2, 64, 100, P, BIG, P, None, P, None] + [P] * 5 + [0.0, P, 0, P, BIG, P, None], **c)


def accept(**c):
    return call("sonic_tree_accept", "B N nodes plan bytes parent token chosen path plen next tokens toff tcap tlen status stream",
                [0, 8, 4, P, BIG] + [P] * 6 + [None] * 4 + [P, None], **c)


def append(**c):
    return call("sonic_cache_append", "B N max Hkv d cu sel slen kn vn kc ks vc vs off cap len status stream",
                [0, 8, 8, 2, 64, P, None, None, P, P, P, None, P, None, P, P, P, P, None], **c)


def logits(**c):
    return call("sonic_logits_process", "B N nodes V x bf16 plan bytes token hist hoff hlen plen rep pres freq bcu btok bval allowed out best "
                "value ws wbytes status stream", [0, 0, 4, 100, P, 0, None, 0] + [None] * 13 + [P, None, P, BIG, P, None], **c)


ALL = [plan, decode, accept, append, logits]
ONE = {plan: dict(B=1), decode: dict(B=1), accept: dict(B=1), append: dict(B=1), logits: dict(B=1, N=1)}


@pytest.mark.parametrize("fn", ALL)
def test_empty_batch_is_done_and_a_missing_status_word_refused(fn):
    assert fn() == sonic.OK
    assert fn(status=None) == sonic.ERR_INVALID_ARG
    assert fn(B=-1) == sonic.ERR_INVALID_ARG
    assert fn(N=-1) == sonic.ERR_INVALID_ARG
    assert fn(B=65536, N=65536 if fn is logits else 8) == sonic.ERR_UNSUPPORTED


@pytest.mark.parametrize("fn", [plan, decode, accept])
def test_plans(fn):
    assert fn(nodes=-1) == sonic.ERR_INVALID_ARG
    assert fn(nodes=257) == sonic.ERR_UNSUPPORTED
    assert fn(B=1, plan=None) == sonic.ERR_INVALID_ARG
    assert fn(B=1, plan=ODD) == sonic.ERR_INVALID_ARG
    for B, N, nodes in ((1, 8, 4), (64, 900, 16), (3, 700, 256)):
        need = sonic.tree_plan_bytes(B, N, nodes)
        assert need >= B * 8 + N * ((nodes + 31) // 32) * 4
        assert fn(B=B, N=N, nodes=nodes, bytes=need - 1) == sonic.ERR_WORKSPACE
    assert sonic.tree_plan_bytes(-1, 8, 4) == 0 and sonic.tree_plan_bytes(1, -8, 4) == 0


def test_logits_on_a_plan():
    need = sonic.tree_plan_bytes(2, 8, 4)
    assert logits(B=2, N=8, plan=P, bytes=need - 1) == sonic.ERR_WORKSPACE
    assert logits(B=2, N=8, plan=P, bytes=BIG, nodes=257) == sonic.ERR_UNSUPPORTED
    assert logits(B=2, N=8) == sonic.ERR_INVALID_ARG          # without one: a row a request
    assert logits(B=2, N=8, nodes=0, plan=P, bytes=BIG) == sonic.OK


@pytest.mark.parametrize("fn", [decode, append])
def test_shapes_that_are_not_supported(fn):
    assert fn(d=96) == sonic.ERR_UNSUPPORTED
    assert fn(Hkv=0) == sonic.ERR_INVALID_ARG


def test_decode_arguments():
    assert decode(Hq=5) == sonic.ERR_INVALID_ARG
    assert decode(Hq=18) == sonic.ERR_UNSUPPORTED             # nine q-heads a kv-head
    assert decode(ctx=-1) == sonic.ERR_INVALID_ARG
    assert decode(ctx=(1 << 30) + 1) == sonic.ERR_UNSUPPORTED and decode(ctx=1 << 30) == sonic.OK
    assert decode(B=65535, Hq=65535, Hkv=65535, N=1 << 30) == sonic.ERR_UNSUPPORTED     # more workgroups than a launch has
    assert decode(ctx=0) == sonic.OK
    assert decode(bf16=2) == sonic.ERR_INVALID_ARG
    for scale in (-1.0, float("nan"), float("inf")):
        assert decode(scale=scale) == sonic.ERR_INVALID_ARG
    assert decode(B=1, N=0) == sonic.OK and decode(B=1, nodes=0) == sonic.OK   # nothing to do
    for n in ("ks", "vs"):
        assert decode(B=1, **{n: P}) == sonic.ERR_INVALID_ARG                  # one tensor's scales
    assert decode(B=1, ks=ODD, vs=P) == sonic.ERR_INVALID_ARG


@pytest.mark.parametrize("fn,names", [(plan, "cu"), (decode, "kc vc off len q kn vn out ws"), (accept, "token chosen path plen next"),
                                      (append, "cu kn vn kc vc off cap len"), (logits, "x ws")])
def test_null_pointers(fn, names):
    for n in names.split():
        assert fn(**ONE[fn], **{n: None}) == sonic.ERR_INVALID_ARG, n


@pytest.mark.parametrize("fn,names", [(decode, "kc vc q kn vn out ws"), (append, "kn vn kc vc"), (logits, "x out allowed ws")])
def test_alignment(fn, names):
    for n in names.split():
        assert fn(**ONE[fn], **{n: ODD}) == sonic.ERR_INVALID_ARG, n


@pytest.mark.parametrize("B,nodes,Hq,Hkv,d,ctx", [(1, 8, 4, 2, 64, 2000), (8, 8, 32, 8, 128, 5000), (1, 64, 32, 8, 128, 100001), (1, 1, 1, 1, 64, 9000)])
def test_small_workspaces(B, nodes, Hq, Hkv, d, ctx):
    need = sonic.tree_decode_workspace_bytes(B, nodes, Hq, d, ctx)
    shape = dict(B=B, N=B * nodes, nodes=nodes, Hq=Hq, Hkv=Hkv, d=d, ctx=ctx)
    assert decode(wbytes=0, **shape) == sonic.ERR_WORKSPACE    # each of these is cut into ranges
    assert need > 256
    for V in (1, 5000, 128000):
        n = sonic.logits_process_workspace_bytes(40, V)
        assert n >= 40 * 8
        assert logits(B=40, N=40, V=V, wbytes=40 * 8 - 1) == sonic.ERR_WORKSPACE
    assert sonic.logits_process_workspace_bytes(-1, 10) == 0 and sonic.logits_process_workspace_bytes(1, -10) == 0


def test_append_and_accept_take_all_of_a_set_or_none():
    for n in ("sel", "slen"):
        assert append(B=1, **{n: P}) == sonic.ERR_INVALID_ARG
    for n in ("ks", "vs"):
        assert append(B=1, **{n: P}) == sonic.ERR_INVALID_ARG
    whole = dict(tokens=P, toff=P, tcap=P, tlen=P)
    for n in whole:
        assert accept(B=1, **{n: P}) == sonic.ERR_INVALID_ARG
        assert accept(B=1, **{**whole, n: None}) == sonic.ERR_INVALID_ARG
    assert append(max=-1) == sonic.ERR_INVALID_ARG


def test_logits_arguments():
    assert logits(V=0) == sonic.ERR_INVALID_ARG
    assert logits(V=(1 << 28) + 1) == sonic.ERR_UNSUPPORTED
    assert logits(bf16=2) == sonic.ERR_INVALID_ARG
    one = dict(B=1, N=1)
    assert logits(**one, best=None) == sonic.ERR_INVALID_ARG   # nothing to write
    assert logits(**one, out=P) == sonic.ERR_INVALID_ARG       # over the logits themselves
    for n in ("hoff", "hlen", "plen", "hist"):
        assert logits(**one, **{n: P}) == sonic.ERR_INVALID_ARG
    assert logits(**one, hist=P, hoff=P) == sonic.ERR_INVALID_ARG
    for n in ("bcu", "btok", "bval"):
        assert logits(**one, **{n: P}) == sonic.ERR_INVALID_ARG


def test_binding_refuses_host_tensors_wrong_types_and_shapes():
    i, bf = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    u = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError):
        sonic.tree_plan(i, None, 4, 4, u, i)
    with pytest.raises(TypeError):
        sonic.tree_plan(i.long(), None, 4, 4, u, i)
    with pytest.raises(TypeError):
        sonic.tree_decode(u, bf, bf, i.long(), i, bf, bf, bf, bf.half(), u, i, 4, 4)
    with pytest.raises(ValueError):
        sonic.tree_decode(u, bf, bf, i.long(), i, bf, bf, bf, bf, u, i, 4, 4, k_scale=u)
    with pytest.raises(TypeError):
        sonic.logits_process(torch.zeros((2, 8), dtype=torch.float16), i, u, i)
    with pytest.raises(ValueError):
        sonic.logits_process(torch.zeros((2, 8)), i, u, i)
    with pytest.raises(ValueError):
        sonic.logits_process(torch.zeros((2, 8)), i[:2], u, i, plan=u)      # without its batch
    with pytest.raises(ValueError):
        sonic.tree_accept(u, None, i, i, i, i, i, i, 4)
    with pytest.raises(ValueError):
        sonic.cache_append(i, bf, bf, bf, bf, i.long(), i, i, i, 4)


# ------------------------------------------------------------------ the oracle
def test_oracle_of_a_chain_is_causal_attention():
    rng = np.random.default_rng(1)
    n, L = 5, 7
    q, k, v, kn, vn = (rng.standard_normal((m, 2, 64)) for m in (n, L, L, n, n))
    out = OT.attend(q, k, v, kn, vn, np.arange(n) - 1)
    for i in range(n):
        kk, vv = np.concatenate([k, kn[:i + 1]]), np.concatenate([v, vn[:i + 1]])
        for h in range(2):
            s = kk[:, h] @ q[i, h] / 8.0
            p = np.exp(s) / np.exp(s).sum()
            assert np.allclose(out[i, h], p @ vv[:, h], rtol=1e-12, atol=1e-12)


def test_oracle_of_paths_and_logits():
    parent, token = [-1, 0, 0, 1, 1, 3, -1], [9, 4, 4, 5, 6, 7, 4]
    assert OT.path_of(parent, 5) == [5, 3, 1, 0]
    assert OT.accepted(parent, token, [4, 5, 1, 7, 0, 8, 2]) == ([0, 1, 3, 5], 8)   # of equal children the first
    assert OT.accepted(parent, token, [3, 5, 1, 7, 0, 8, 2]) == ([0], 3)
    x, best, value = OT.logits_row(np.array([2.0, 2.0, -1.0, 2.0]), [1], [2, 2], 2.0, 0.5, 0.25, [(3, 9.0), (3, -1.0)], None)
    assert x.tolist() == [2.0, 1.0, -3.0, 1.0] and (best, value) == (0, 2.0)
    assert OT.logits_row(np.array([2.0, np.nan]), [], [], 1, 0, 0, [], np.array([False, True]))[1] == -1
