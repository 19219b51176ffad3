"""Steps over drafted tokens and eviction on one cache: an append knows nothing of row weights, its caller sets those of the rows
that it wrote, on the device, and the next eviction goes by them."""
import numpy as np
import pytest
import torch

from oracle import evict as OE
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import bf16_to_device
from tests import gpu_helpers as H
from tests.test_gpu_decode_exact import set_rows
from tests.test_gpu_q4 import Cache, i32
from tests.test_gpu_tree import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q4", [False, True])
def test_appended_rows_are_weighed(q4):
    H.need_gpu()
    rng = np.random.default_rng(51 + q4)
    lens, nodes, B = [40, 7, 300, 0], [5, 3, 9, 2], 4
    c = Cache(rng, lens, 12, 2, 64, q4)
    dev = c.dev
    dev.keep_idx.copy_(dev.place)
    request = torch.repeat_interleave(torch.arange(B, device="cuda"), i32(c.cap).long())
    budget = i32([20, 100, 64, 1])
    # the rows that each request holds: (bits of k, bits of v, weight, position)
    held = [[(c.bits[0][o + j], c.bits[1][o + j], c.weight[o + j], j) for j in range(n)] for o, n in zip(c.off, lens)]
    for turn in range(3):
        s = Step(rng, c, 4, nodes)
        assert s.step.plan_trees(i32(s.cu), s.parent, s.status) == sonic.OK
        chosen = rng.integers(0, 2, s.N)
        token = rng.integers(0, 2, s.N)
        assert s.step.accept(s.parent, i32(token), s.status, chosen=i32(chosen)) == sonic.OK
        old = dev.length.clone()
        assert dev.append(i32(s.cu), bf16_to_device(s.k), bf16_to_device(s.v), s.status, s.step.max_nodes, select=s.step.path,
                          select_len=s.step.path_len) == sonic.OK
        # the caller's part: a weight and a position for every new row, without a look at the lengths on the host
        new = (dev.place >= old[request]) & (dev.place < dev.length[request])
        dev.row_weight.copy_(torch.where(new, 0.25 * (turn + 1), dev.row_weight))
        dev.keep_idx.copy_(torch.where(new, 1000 * (turn + 1) + dev.place - old[request], dev.keep_idx))
        assert dev.evict(i32([2] * B), i32([1] * B), budget, s.status) == sonic.OK
        torch.cuda.synchronize()
        assert int(s.status.item()) == 0
        path, m = s.step.path.cpu().numpy(), s.step.path_len.tolist()
        weight, keep = dev.row_weight.cpu().numpy(), dev.keep_idx.cpu().numpy()
        for b in range(B):
            held[b] += [(s.k[i], s.v[i], np.float32(0.25 * (turn + 1)), 1000 * (turn + 1) + j)
                        for j, i in enumerate(s.cu[b] + path[s.cu[b]:s.cu[b] + m[b]])]
            stay = OE.kept_rows([x[2] for x in held[b]], 2, 1, int(budget[b]))
            held[b] = [held[b][i] for i in stay]
            o = int(c.off[b])
            assert int(dev.length[b]) == len(held[b]) and m[b] >= 1
            assert np.array_equal(weight[o:o + len(held[b])], [x[2] for x in held[b]])
            assert np.array_equal(keep[o:o + len(held[b])], [x[3] for x in held[b]])
    # what is held is what the next step attends to
    want = Cache(rng, [len(x) for x in held], 12, 2, 64, q4)
    for b, rows in enumerate(held):
        o = int(want.off[b])
        for j, x in enumerate(rows):
            want.bits[0][o + j], want.bits[1][o + j] = x[0], x[1]
    set_rows(want, *want.bits)
    s = Step(rng, want, 4, nodes)
    expected = s.run()
    s.check(expected)
    s.c = c
    assert np.array_equal(s.run(max_ctx=s.max_ctx), expected)
