"""Host bounds at the largest number they can be: a caller that knows no better one gets the same results."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import q4 as OQ
from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_evict import Rows, i32
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("q4", [True, False])
def test_compaction_and_key_weights(q4):
    H.need_gpu()
    rng = np.random.default_rng(81)
    lays = [W.RequestLayout(30, [700, 900], [600, 20], 1500), W.RequestLayout(5, [100], [40], 17)]
    batch = W.make_batch("bounds", lays, 2, 2, 64, seed=81)
    db = H.device_batch(batch)
    caps = H.kept_counts(batch) + 2
    cache = db.alloc_cache_q4(caps) if q4 else db.alloc_cache(caps)
    db.max_seqlen = MOST
    assert (db.compact_q4() if q4 else db.compact()) == sonic.OK
    assert db.read_status() == 0 and np.array_equal(cache.length.cpu().numpy(), H.kept_counts(batch))
    kc, vc, idx, _, _ = H.oracle_compact(batch, caps)
    assert np.array_equal(cache.keep_idx.cpu().numpy(), idx)
    if q4:
        assert np.array_equal(cache.k.cpu().numpy()[idx >= 0], OQ.pack(OQ.encode(kc[idx >= 0])[0]))
    key_weight, rw = torch.rand(batch.total_tokens, device="cuda"), torch.full((cache.k.shape[0],), -1.0, device="cuda")
    assert sonic.kv_compact_weights(db.cu, key_weight, cache.row_off, cache.length, cache.keep_idx, rw, db.status, MOST) == sonic.OK
    kw, want = key_weight.cpu().numpy(), np.full(len(idx), -1.0, np.float32)
    for b, (o, n) in enumerate(zip(cache.row_off_host, H.kept_counts(batch))):
        want[o:o + n] = kw[batch.cu_seqlens[b] + idx[o:o + n]]
    assert db.read_status() == 0 and np.array_equal(rw.cpu().numpy(), want)


def test_expansion():
    H.need_gpu()
    c = Cache(np.random.default_rng(82), [500, 0, 37], 2, 3, 128, True)
    out = torch.zeros((2, int(c.cap.sum()), 3, 128), dtype=torch.bfloat16, device="cuda")
    assert c.dev.expand(i32([0, 0, 0]), c.dev.length, out[0], out[1], c.dev.row_off, c.dev.row_cap, c.status, MOST) == sonic.OK
    assert int(c.status.item()) == 0
    for got, values in zip(out.double().cpu().numpy(), c.values):
        for o, n in zip(c.off, c.lens):
            assert np.array_equal(got[o:o + n], values[o:o + n])


@pytest.mark.parametrize("q4,weighted", [(True, False), (True, True), (False, True)])
def test_decode(q4, weighted):
    """The weighted forms' workspace holds a score per head and row of the bound, 8 GiB here."""
    H.need_gpu()
    rng = np.random.default_rng(83)
    c = Cache(rng, [3000], 2, 1, 64, q4)
    c.check(*c.step(rng, 1, weighted=weighted, max_ctx=MOST), weighted=weighted)


@pytest.mark.parametrize("q4", [True, False])
def test_eviction(q4):
    H.need_gpu()
    r = Rows(np.random.default_rng(84), [9000], 1, 1, 64, q4)
    kept = r.kept(5, 6, 700)[0]
    a, kw = r.args(5, 6, 700)
    ws = torch.empty(sonic.cache_evict_workspace_bytes(1, MOST), dtype=torch.uint8, device="cuda")
    assert sonic.cache_evict(*a[:-3], ws, r.status, MOST, **kw) == sonic.OK
    assert int(r.status.item()) == 0 and r.length.tolist() == [700]
    assert np.array_equal(r.row_weight.cpu().numpy()[:700], r.weight[kept])
    for name, x in r.host.items():
        assert np.array_equal(r.bytes(name)[:700], x[kept])
