"""What a tree attention's workspace held before the call does not reach its outputs: contents need no initialisation, and a
call that was stopped leaves marks for its own ranges only.  Shapes in several ranges whose rows do not fill the last
workgroup of the join, so that some of its threads stand past the request's rows."""
import numpy as np
import pytest
import torch

from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_q4 import Cache
from tests.test_gpu_tree import Step

pytestmark = pytest.mark.gpu

SHAPES = [([5000], 4, 2, 64, [3]), ([2000], 4, 2, 64, [1]), ([8000], 28, 4, 128, [13]), ([8000], 8, 8, 128, [13]),
          ([6000, 40, 4100], 6, 2, 64, [5, 9, 1])]


def make(seed, lens, Hq, Hkv, d, nodes, q4):
    """A call, and its workspace."""
    s = Step(np.random.default_rng(seed), Cache(np.random.default_rng(seed + 1), lens, 1, Hkv, d, q4), Hq, nodes)
    n = sonic.tree_decode_workspace_bytes(len(lens), max(nodes), Hq, d, max(lens))
    assert n > 1024                                         # in ranges
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    s.c.dev.workspaces.made["tree"] = [ws]
    return s, ws


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,d,nodes", SHAPES)
def test_any_contents(lens, Hq, Hkv, d, nodes, q4, out):
    """-infinity, as masked scores leave it (and as a stopped range is marked), NaN, and negative numbers."""
    H.need_gpu()
    s, ws = make(sum(lens) + d + q4, lens, Hq, Hkv, d, nodes, q4)
    want = None
    for word in (0.0, -np.inf, np.nan, -1.0):
        ws.view(torch.float32).fill_(float(word))
        got = s.run(out)
        s.check(got, out)
        want = got if want is None else want
        assert np.array_equal(got, want), word


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,d,nodes", SHAPES)
def test_a_call_behind_a_stopped_one(lens, Hq, Hkv, d, nodes, q4, out):
    H.need_gpu()
    s, ws = make(sum(lens) + d + q4, lens, Hq, Hkv, d, nodes, q4)
    ws.zero_()
    want = s.run(out)
    s.check(want, out)
    s.status.fill_(sonic.ERR_BAD_LAYOUT)
    assert np.all(s.run(out) == 7.0)
    s.status.zero_()
    assert np.array_equal(s.run(out), want)
