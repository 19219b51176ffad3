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


def test_a_dead_end_confirms_no_padding():
    """A row whose mask leaves nothing has -1 for its best token, and trees may be padded with nodes of token -1: the path ends
    there, and neither the history nor the cache gets a padding row."""
    H.need_gpu()
    status = i32([0])
    nodes, V = [4, 3, 70], 40
    cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    n = int(cu[-1])
    parents = [[-1, 0, 1, 1], [-1, 0, 1], [-1] + list(range(69))]
    token = np.full(n, -1)                                    # all padding, but for ..
    token[:2], token[4:6], token[7] = (5, 9), (3, 6), 8       # .. 5 -> 9; 3 -> 6; 8
    logits = torch.zeros((n, V), device="cuda")
    logits[0, 9] = logits[4, 6] = logits[5, 2] = 1.0
    allowed = np.zeros((n, 64), np.uint8)
    allowed[:, :V] = 1
    allowed[1] = allowed[7] = 0                               # nothing behind 9, nothing behind 8
    allowed = torch.from_numpy(np.packbits(allowed, axis=1, bitorder="little").view(np.int32)).cuda()
    step = DraftStep(3, n, 70)
    parent = i32(np.concatenate(parents))
    assert step.plan_trees(i32(cu), parent, status) == sonic.OK
    assert step.logits(logits, status, allowed=allowed) == sonic.OK
    assert step.best[[0, 1, 4, 5, 7]].tolist() == [9, -1, 6, 2, -1]
    history = dict(tokens=i32([0] * 300), token_off=torch.tensor([0, 100, 200], device="cuda"), token_cap=i32([100] * 3), token_len=i32([4] * 3))
    assert step.accept(parent, i32(token), status, **history) == sonic.OK
    c = Cache(np.random.default_rng(6), [10, 20, 30], 70, 2, 64, False)
    x = bf16_to_device(normal_bits(np.random.default_rng(7), n, 2, 64))
    assert c.dev.append(i32(cu), x, x, status, 70, select=step.path, select_len=step.path_len) == sonic.OK
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert step.path_len.tolist() == [2, 2, 1] and step.next_token.tolist() == [-1, 2, -1]
    assert step.path[:7].tolist() == [0, 1, -1, -1, 0, 1, -1] and step.path[7:].tolist() == [0] + [-1] * 69
    assert history["token_len"].tolist() == [6, 6, 5] and c.dev.length.tolist() == [12, 22, 31]
    assert history["tokens"].tolist()[4:7] == [5, 9, 0] and history["tokens"].tolist()[204:206] == [8, 0]


@pytest.mark.parametrize("choice", [-1, -2, -2 ** 31])
def test_negative_choices_of_a_sampler(choice):
    """.. end the path too, and are what the caller is given back."""
    H.need_gpu()
    status, step = i32([0]), DraftStep(1, 3, 3)
    assert step.plan_trees(i32([0, 3]), None, status) == sonic.OK
    assert step.accept(None, i32([1, choice, choice]), status, chosen=i32([choice] * 3)) == sonic.OK
    assert step.path_len.tolist() == [1] and step.next_token.tolist() == [choice] and step.path.tolist() == [0, -1, -1]


@pytest.mark.parametrize("nodes", [4, 100])
@pytest.mark.parametrize("cu,parent,most,rows", [([1, 2, 4], [-1] * 4, 4, slice(0, 2)), ([0, 2, 5], [-1] * 4, 4, slice(2, 4)),
                                                 ([0, 3, 4], [-1] * 4, 2, slice(0, 2)), ([0, 2, 4], [-1, 1, -1, 0], 4, slice(0, 2)),
                                                 ([0, 2, 4], [-1, 0, -2, 0], 4, slice(2, 4)), ([0, 2, 4], [-1, 0, -1, 7], 4, slice(2, 4))])
def test_a_request_with_a_malformed_tree_has_no_rows(cu, parent, most, rows, nodes):
    """.. whatever its caller does about the status word: attention, best tokens and path leave its rows as they were."""
    H.need_gpu()
    nodes = most if most < 4 else nodes
    c = Cache(np.random.default_rng(3), [30, 300], 1, 2, 64, False)
    step = DraftStep(2, 4, nodes)
    whole = step.plan_trees(i32([0, 2, 4]), None, c.status)            # an earlier step's plan
    assert whole == sonic.OK and step.plan_trees(i32(cu), i32(parent), c.status) == sonic.OK
    assert int(c.status.item()) == sonic.ERR_BAD_LAYOUT
    c.status.zero_()
    q, x = (torch.zeros((4, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    out, best = torch.full((4, 4, 64), 7.0, device="cuda"), torch.full((4,), -7, dtype=torch.int32, device="cuda")
    assert c.dev.tree_decode(step.plan, q, x, x, out, c.status, nodes, 300) == sonic.OK
    step.best.fill_(-7)
    step.path.fill_(-9)
    assert step.logits(torch.zeros((4, 50), device="cuda"), c.status) == sonic.OK
    assert step.accept(i32(parent), best, c.status) == sonic.OK
    torch.cuda.synchronize()
    assert torch.all(out[rows] == 7.0) and torch.all(step.best[rows] == -7) and torch.all(step.path[rows] == -9)


@pytest.mark.parametrize("q4", [False, True])
def test_a_cache_without_room_is_brought_up_to_its_history(q4):
    """A path that its history had room for and one cache had not: that cache alone stays behind, its rows are told by the lengths,
    and a later append of that request's path alone brings it up."""
    H.need_gpu()
    rng = np.random.default_rng(8)
    nodes = [3, 4, 2]
    cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    caches = [Cache(rng, [10, 20, 30], 4, 2, 64, q4) for _ in range(2)]
    caches[1].dev.row_cap[1] = 21                             # of the second layer, request 1: one row left
    status, step = i32([0]), DraftStep(3, 9, 4)
    bits = [[normal_bits(rng, 9, 2, 64) for _ in range(2)] for _ in caches]
    history = dict(tokens=i32([0] * 60), token_off=torch.tensor([0, 20, 40], device="cuda"), token_cap=i32([20] * 3), token_len=i32([10] * 3))
    before = [c.dev.length.clone() for c in caches]
    rows = [rows_of(c) for c in caches]
    assert step.plan_trees(i32(cu), None, status) == sonic.OK
    assert step.accept(None, i32([5] * 9), status, chosen=i32([5, 5, 0, 5, 5, 5, 0, 0, 0]), **history) == sonic.OK
    for c, x in zip(caches, bits):
        assert c.dev.append(i32(cu), *(bf16_to_device(y) for y in x), status, 4, select=step.path, select_len=step.path_len) == sonic.OK
    assert int(status.item()) == sonic.ERR_CAPACITY
    assert step.path_len.tolist() == [3, 4, 1] and history["token_len"].tolist() == [13, 14, 11]
    assert caches[0].dev.length.tolist() == [13, 24, 31] and caches[1].dev.length.tolist() == [13, 20, 31]
    # with room, the path of the requests that stayed behind, and of no other
    status.zero_()
    caches[1].dev.row_cap[1] = 24
    for c, x, n in zip(caches, bits, before):
        behind = torch.where(c.dev.length == n, step.path_len, 0).int()
        assert c.dev.append(i32(cu), *(bf16_to_device(y) for y in x), status, 4, select=step.path, select_len=behind) == sonic.OK
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for c, x, r in zip(caches, bits, rows):
        assert c.dev.length.tolist() == [13, 24, 31]
        for b, m in enumerate([3, 4, 1]):
            for j in range(m):
                put(c, r, int(c.off[b] + c.lens[b]) + j, [y[cu[b] + j] for y in x])
        assert all(np.array_equal(a, b) for a, b in zip(rows_of(c), r))
