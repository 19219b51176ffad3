"""What the calls over cache rows leave when one of their requests is at fault: every other request's rows are written,
however the workgroups come to run."""
import numpy as np
import pytest
import torch

from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import Q4Cache
from tests import gpu_helpers as H

pytestmark = pytest.mark.gpu

B, ROWS = 3000, 300


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("begin,end,cap,max_rows,code", [(-1, ROWS, ROWS, ROWS, sonic.ERR_BAD_LAYOUT), (0, ROWS + 1, ROWS, ROWS + 1, sonic.ERR_BAD_LAYOUT),
                                                         (0, ROWS, ROWS - 1, ROWS, sonic.ERR_CAPACITY), (0, ROWS, ROWS, ROWS - 1, sonic.ERR_INVALID_ARG)])
@pytest.mark.parametrize("at", [0, B - 1])
def test_expansion_writes_every_request_but_the_one_at_fault(at, begin, end, cap, max_rows, code):
    H.need_gpu()
    off = np.arange(B, dtype=np.int64) * ROWS
    c = Q4Cache(B * ROWS, 1, 64, off, np.full(B, ROWS), "cuda")
    for x in (c.k, c.v):
        x.fill_(0x22)                 # 1.0 under the scale below
    for x in (c.k_scale, c.v_scale):
        x.fill_(127)
    begins, ends, caps = np.zeros(B, int), np.full(B, min(max_rows, ROWS)), np.full(B, ROWS)
    begins[at], ends[at], caps[at] = begin, end, cap
    k, v = (torch.full((B, ROWS, 1, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    status = i32([0])
    st = c.expand(i32(begins), i32(ends), k.view(-1, 1, 64), v.view(-1, 1, 64), c.row_off, i32(caps), status, max_rows)
    assert st == sonic.OK and int(status.item()) == code
    n = min(max_rows, ROWS)
    others = torch.arange(B, device="cuda") != at
    for x in (k, v):
        assert bool((x[others, :n] == 1.0).all()) and bool((x[others, n:] == 5.0).all())
        assert bool((x[at] == 5.0).all())


def weights_call(c, key_weight, cu, status, max_rows=ROWS):
    return sonic.kv_compact_weights(cu, key_weight, c.row_off, c.length, c.keep_idx, c.row_weight, status, max_rows)


@pytest.mark.parametrize("fault,code", [("index", sonic.ERR_BAD_LAYOUT), ("negative index", sonic.ERR_BAD_LAYOUT), ("length", sonic.ERR_INVALID_ARG),
                                        ("negative length", sonic.ERR_BAD_LAYOUT)])
@pytest.mark.parametrize("at", [0, B - 1])
def test_key_weights_reach_every_row_but_those_at_fault(at, fault, code):
    H.need_gpu()
    cap = ROWS + 1
    c = Q4Cache(B * cap, 1, 64, np.arange(B, dtype=np.int64) * cap, np.full(B, cap), "cuda")
    c.length.fill_(ROWS)
    c.keep_idx.copy_(torch.arange(B * cap, device="cuda") % cap)
    c.row_weight.fill_(-1.0)
    key_weight = torch.rand(B * ROWS, device="cuda")
    cu = i32(np.arange(B + 1) * ROWS)
    want = torch.full((B, cap), -1.0, device="cuda")
    want[:, :ROWS] = key_weight.view(B, ROWS)
    if "index" in fault:
        c.keep_idx[at * cap + 7] = ROWS if fault == "index" else -1
        want[at, 7] = -1.0
    else:
        c.length[at] = ROWS + 1 if fault == "length" else -1
        want[at] = -1.0
    status = i32([0])
    assert weights_call(c, key_weight, cu, status) == sonic.OK
    assert int(status.item()) == code
    assert torch.equal(c.row_weight.view(B, cap), want)
    # a status that was pending before the call stops it
    c.row_weight.fill_(-1.0)
    assert weights_call(c, key_weight, cu, status) == sonic.OK
    assert int(status.item()) == code and bool((c.row_weight == -1.0).all())
