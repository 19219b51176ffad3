"""After an eviction through the cache classes every row still names the prompt position that it came from."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import evict as OE
from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_evict import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q4", [True, False])
def test_positions_and_key_weights_after_an_eviction(q4):
    H.need_gpu()
    rng = np.random.default_rng(61 + q4)
    lays = [W.random_layout(rng, max_h=4, max_b=300, max_k=90, max_s=60, max_c=60) for _ in range(5)] + [W.RequestLayout(0, [], [], 0),
                                                                                                         W.RequestLayout(40, [200], [300], 9)]
    batch = W.make_batch("positions", lays, 4, 2, 64, seed=61)
    db = H.device_batch(batch)
    caps = H.kept_counts(batch) + 2
    cache = db.alloc_cache_q4(caps) if q4 else db.alloc_cache(caps)
    assert (db.compact_q4() if q4 else db.compact()) == sonic.OK
    key_weight = torch.rand(batch.total_tokens, device="cuda")
    cache.row_weight = torch.zeros(cache.k.shape[0], device="cuda")

    def weigh():
        st = sonic.kv_compact_weights(db.cu, key_weight, cache.row_off, cache.length, cache.keep_idx, cache.row_weight, db.status, int(caps.max()))
        assert st == sonic.OK and db.read_status() == 0
        return cache.row_weight.cpu().numpy()

    kw = key_weight.cpu().numpy()
    pos = [cache.keep_idx[o:o + n].cpu().numpy() for o, n in zip(cache.row_off_host, H.kept_counts(batch))]
    for budget in (150, 60):
        w = weigh()
        before = cache.keep_idx.clone()
        db.status.fill_(sonic.ERR_CAPACITY)          # a call that is refused moves nothing
        lim = [i32([x] * len(lays)) for x in (4, 3, budget)]
        assert cache.evict(*lim, db.status) == sonic.OK
        assert torch.equal(cache.keep_idx, before)
        db.clear_status()
        assert cache.evict(*lim, db.status) == sonic.OK and db.read_status() == 0
        got = cache.keep_idx.cpu().numpy()
        for b, o in enumerate(cache.row_off_host):
            pos[b] = pos[b][OE.kept_rows(w[o:o + len(pos[b])], 4, 3, budget)]
            assert np.array_equal(got[o:o + len(pos[b])], pos[b])
            assert np.array_equal(got[o + len(pos[b]):o + caps[b]], before[o + len(pos[b]):o + caps[b]].cpu().numpy())
        cache.row_weight.fill_(-1.0)
        w = weigh()
        for b, o in enumerate(cache.row_off_host):
            assert np.array_equal(w[o:o + len(pos[b])], kw[batch.cu_seqlens[b] + pos[b]])
        assert (w == -1.0).sum() == len(w) - sum(map(len, pos))
