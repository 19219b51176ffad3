"""One decode workspace for calls of several bounds, head dims and forms: zeroed once for its batch and kv-heads."""
import numpy as np
import pytest
import torch

from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("B,Hkv,lens", [(3, 2, [100, 900, 17]), (40, 8, [2100] + [30, 4, 17] * 13)])
def test_a_workspace_serves_other_bounds_heads_and_forms(B, Hkv, lens, q4):
    H.need_gpu()
    rng = np.random.default_rng(B + q4)
    shapes = [(2 * Hkv, 64, 3000), (Hkv, 128, 2200), (4 * Hkv, 64, 2110), (2 * Hkv, 128, 5000)]
    size = (lambda hq, d, n: sonic.decode_q4_workspace_bytes(B, hq, d, n, True)) if q4 else \
        (lambda hq, d, n: sonic.decode_weighted_workspace_bytes(B, hq, d, n))
    ws = torch.zeros(max(size(*s) for s in shapes), dtype=torch.uint8, device="cuda")
    for Hq, d, bound in shapes + shapes[::-1]:
        for weighted in (True, False):
            c = Cache(rng, lens, 2, Hkv, d, q4)
            dev = c.dev

            def decode(q, k, v, out, status, max_ctx, weighted=weighted):
                rows = (dev.row_off, dev.row_cap, dev.length, q, k, v, out)
                if q4:
                    return sonic.compressed_decode_q4(dev.k, dev.k_scale, dev.v, dev.v_scale, *rows, ws, status, max_ctx,
                                                      row_weight=dev.row_weight if weighted else None)
                if weighted:
                    return sonic.compressed_decode_weighted(dev.k, dev.v, *rows, dev.row_weight, ws, status, max_ctx)
                return sonic.compressed_decode(dev.k, dev.v, *rows, ws, status, max_ctx)

            dev.decode = decode
            dev.decode_weighted = decode
            if q4:
                step = c.step(rng, Hq, weighted=weighted, max_ctx=bound)
            else:
                step = c.step(rng, Hq, max_ctx=bound)
            assert int(c.status.item()) == 0
            if q4 or weighted:
                c.check(*step, weighted=weighted)
            else:
                for b in range(B):
                    H.assert_close(step[3][b], c.expect(b, *step[:3])[0], f"request {b}")
