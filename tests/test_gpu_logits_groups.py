"""Logits of trees whose workgroups have several rows each: the request's table is made once for them, a row's path is added
and taken off again, and the next row's logits, with other places in the 16-byte parts, are on their way during the stores."""
import numpy as np
import pytest
import torch

from oracle import tree as OT
from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_logits import Call

pytestmark = pytest.mark.gpu


def group_of(B, most, V):
    """Rows of a workgroup (the library's rule: pieces of 4,096 tokens, some 1,024 workgroups)."""
    return max(1, min(most, (V + 4095) // 4096 * B * most // 1024))


def paths_share_tokens(c, rng, few):
    """Path tokens from a few, several times on a path, many of them in the prompt, the answer and the biases too, at the ends of
    pieces among others."""
    ends = [x for x in (0, 4095, 4096, c.V - 1, c.V // 2) if x < c.V]
    some = np.concatenate([ends, rng.integers(0, c.V, max(1, few - len(ends)))]).astype(np.int32)
    c.node_token[:] = rng.choice(some, len(c.node_token))
    for x in (c.tokens, c.bias_token):
        at = rng.random(len(x)) < 0.5
        x[at] = rng.choice(some, int(at.sum()))
    for b in range(c.B):                      # of every tree, a token that a path holds at least twice where it is long enough
        for i in range(len(c.parents[b])):
            path = OT.path_of(c.parents[b], i)
            if len(path) > 2:
                c.node_token[c.cu[b] + path[2]] = c.node_token[c.cu[b] + i]
                break


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V,nodes,group", [(50257, [33, 1, 7, 20, 32, 2, 0, 31], 3), (60001, [24, 23, 5, 1] * 4, 5),
                                           (20001, [2, 1, 0] * 100, 2), (128000, [32, 31, 9, 1, 30, 32, 17, 8], 8),
                                           (50258, [64, 40, 3, 63, 50, 1], 4)])
def test_rows_of_one_workgroup(V, nodes, group, bf16):
    """Odd and even vocabularies, groups that the requests' rows do not fill."""
    H.need_gpu()
    assert group_of(len(nodes), max(nodes), V) == group and any(n % group for n in nodes)
    rng = np.random.default_rng(V + group + bf16)
    c = Call(rng, len(nodes), V, bf16, nodes=nodes, hist=60, biases=12)
    paths_share_tokens(c, rng, 12)
    c.run().check()


@pytest.mark.parametrize("parts,biases,mask", [(("path",), 0, None), (("path", "penalties"), 0, "few"), (("history", "penalties"), 5, None)])
def test_rows_of_one_workgroup_without_some_parts(parts, biases, mask):
    H.need_gpu()
    nodes, V = [33, 1, 7, 20, 32, 2, 0, 31], 50257
    assert group_of(len(nodes), max(nodes), V) == 3
    rng = np.random.default_rng(len(parts) + biases)
    c = Call(rng, len(nodes), V, nodes=nodes, hist=60, biases=biases, mask=mask, parts=parts)
    paths_share_tokens(c, rng, 9)
    c.run().check()
    want = c.best.clone()
    c.run(out=False).check()
    assert torch.equal(c.best, want)


def test_bias_ranges_that_run_backwards():
    """Nothing is written for the request whose range ends before it starts; the next one's begins there, and is done."""
    H.need_gpu()
    for nodes in (None, [2, 3, 2, 1]):
        rng = np.random.default_rng(13)
        c = Call(rng, 4, 5000, nodes=nodes)
        c.bias_cu = np.array([0, 2, 5, 4, 10], np.int32)
        c.bias_token, c.bias_value = rng.integers(0, 5000, 10).astype(np.int32), rng.standard_normal(10).astype(np.float32)
        c.parts.add("biases")
        c.run()
        assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
        c.check(skip=(2,))
