"""What the calls of a step over drafted tokens do about errors: a pending capacity error, which stops nothing, hides no other
one, and the requests that are not at fault are done."""
import numpy as np
import pytest
import torch

from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import DraftStep, bf16_to_device
from tests import gpu_helpers as H
from tests.test_gpu_logits import Call
from tests.test_gpu_q4 import Cache, i32, normal_bits
from tests.test_gpu_tree_step import put, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [4, 100])
@pytest.mark.parametrize("cu,parent", [([0, 3, 2], [-1, 0, 0, 0]), ([0, 2, 4], [-1, 1, -1, 0]), ([0, 2, 4], [-1, 0, -2, 0])])
def test_a_malformed_tree_behind_a_capacity_error(cu, parent, nodes):
    """The plan's error stands in the status word, and the calls behind it write nothing."""
    H.need_gpu()
    c = Cache(np.random.default_rng(1), [30, 300], 1, 2, 64, False)
    step = DraftStep(2, 4, nodes)
    c.status.fill_(sonic.ERR_CAPACITY)
    assert step.plan_trees(i32(cu), i32(parent), c.status) == sonic.OK
    assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
    out = torch.full((4, 4, 64), 7.0, device="cuda")
    q, x = (torch.zeros((4, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    assert c.dev.tree_decode(step.plan, q, x, x, out, c.status, nodes, 300) == sonic.OK
    assert torch.all(out == 7.0) and int(c.status.item()) == sonic.ERR_BAD_LAYOUT


@pytest.mark.parametrize("nodes", [None, [2, 3, 2, 1]])
def test_a_bad_history_behind_a_capacity_error(nodes):
    H.need_gpu()
    c = Call(np.random.default_rng(2), 4, 5000, nodes=nodes)
    c.len[2] = -1
    c.status.fill_(sonic.ERR_CAPACITY)
    c.run()
    assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
    c.check(skip=(2,))


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("pending", [sonic.OK, sonic.ERR_CAPACITY])
@pytest.mark.parametrize("full,fault", [(1, 6), (6, 1), (4, 300), (300, 4), (None, 2)])
def test_a_bad_append_beside_a_full_cache(full, fault, pending, q4):
    """One request without room and one with a bad selection, in either order and far from each other, or a capacity error from
    a call before: the selection's error is what the status word says, and the other requests get their rows."""
    H.need_gpu()
    rng = np.random.default_rng(3)
    B, m = 301, 2
    c = Cache(rng, [4] * B, m, 2, 64, q4)
    bits = [normal_bits(rng, B * m, 2, 64) for _ in range(2)]
    select = np.tile(np.arange(m), B)
    select[fault * m + 1] = m
    if full is not None:
        c.dev.row_cap[full] = 5
    c.status.fill_(pending)
    rows = rows_of(c)
    assert c.dev.append(i32(np.arange(B + 1) * m), *(bf16_to_device(x) for x in bits), c.status, m, select=i32(select),
                        select_len=i32([m] * B)) == sonic.OK
    assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
    for b in range(B):
        for j in range(m if b not in (full, fault) else 0):
            put(c, rows, int(c.off[b]) + 4 + j, [x[b * m + j] for x in bits])
    assert all(np.array_equal(x, y) for x, y in zip(rows_of(c), rows))
    assert c.dev.length.tolist() == [4 if b in (full, fault) else 4 + m for b in range(B)]


def test_too_many_rows_behind_a_capacity_error_and_capacity_behind_others():
    H.need_gpu()
    c = Cache(np.random.default_rng(4), [4, 5], 6, 2, 64, False)
    x = bf16_to_device(normal_bits(np.random.default_rng(5), 4, 2, 64))
    c.status.fill_(sonic.ERR_CAPACITY)
    assert c.dev.append(i32([0, 1, 4]), x, x, c.status, 2) == sonic.OK          # three rows, of two at most
    assert int(c.status.item()) == sonic.ERR_INVALID_ARG and c.dev.length.tolist() == [5, 5]
    for code in (sonic.ERR_CAPACITY, sonic.ERR_BAD_LAYOUT, sonic.ERR_INVALID_ARG):
        c.status.fill_(code)
        c.dev.row_cap.copy_(i32([1, 1]))
        assert c.dev.append(i32([0, 1, 4]), x, x, c.status, 3) == sonic.OK
        assert int(c.status.item()) == code
