"""Eviction behind an error of an earlier call: a length may be anything then, and no row is looked at for it."""
import numpy as np
import pytest
import torch

from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_evict import Rows, away_cache, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("away", [False, True])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("B,garbage", [(3, 52), (3, -7), (3, 2 ** 31 - 1), (70, 52)])
def test_lengths_behind_a_pending_error_are_not_read(B, garbage, q4, away):
    H.need_gpu()
    r = Rows(np.random.default_rng(51), [50] + [4] * (B - 1), 2, 2, 64, q4)
    r.length[1:] = garbage                  # 52: within the host bound, far past what the requests own
    r.status.fill_(sonic.ERR_BAD_LAYOUT)
    out, _, more = away_cache(r, np.full(B, 52))
    a, kw = r.args(1, 1, 3)
    assert sonic.cache_evict(*a, **kw, **(more if away else {})) == sonic.OK
    torch.cuda.synchronize()
    assert int(r.status.item()) == sonic.ERR_BAD_LAYOUT
    for name, x in r.host.items():
        assert np.array_equal(r.bytes(name), x) and not out[name].view(torch.uint8).any()
    assert np.array_equal(r.row_weight.cpu().numpy(), r.weight)
    assert r.length.tolist() == [50] + [garbage] * (B - 1) and torch.all(more["out_len"] == -5)
    # and the next call, with all in order
    r.status.zero_()
    r.length.copy_(i32(r.lens))
    assert sonic.cache_evict(*a, **kw) == sonic.OK
    assert int(r.status.item()) == 0 and r.length.tolist() == [3] * B


@pytest.mark.parametrize("q4", [False, True])
def test_a_status_word_that_changes_while_evictions_run(q4):
    """Each request is done as a whole or left as it is."""
    H.need_gpu()
    rng = np.random.default_rng(52)
    lens = [300, 20, 900, 5, 4000, 60] * 8
    r = Rows(rng, lens, 0, 1, 64, q4)
    flips = H.Flips(r.status, sonic.ERR_BAD_LAYOUT)
    a, kw = r.args(2, 2, 50)
    kept = r.kept(2, 2, 50)
    start = {n: x.clone() for n, x in r.dev.items()}
    w0, l0 = r.row_weight.clone(), r.length.clone()
    results = []
    flips.start()
    for _ in range(10):
        for n, x in start.items():
            r.dev[n].copy_(x)
        r.row_weight.copy_(w0)
        r.length.copy_(l0)
        assert sonic.cache_evict(*a, **kw) == sonic.OK
        results.append([r.length.clone(), r.row_weight.clone(), r.dev["k"].clone(), r.dev["v"].clone()])
    torch.cuda.synchronize()
    for length, weight, k, v in results:
        for b, (o, n) in enumerate(zip(r.off, lens)):
            done = int(length[b]) != n
            rows = torch.from_numpy(np.concatenate([kept[b], np.arange(len(kept[b]), n)]) if done else np.arange(n)).cuda() + int(o)
            assert not done or int(length[b]) == len(kept[b])
            assert torch.equal(weight[o:o + n], w0[rows])
            assert torch.equal(k[o:o + n].view(torch.uint8), start["k"][rows].view(torch.uint8))
            assert torch.equal(v[o:o + n].view(torch.uint8), start["v"][rows].view(torch.uint8))
