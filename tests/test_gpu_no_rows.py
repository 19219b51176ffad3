"""Compactions of batches without tokens into caches without rows (empty tensors, whose pointers are null)."""
import pytest
import torch

from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_both_compactions_take_a_batch_without_tokens_or_rows(d):
    H.need_gpu()
    empty = lambda *shape, t=torch.uint8: torch.zeros(shape, dtype=t, device="cuda")
    cu, cap, off = empty(4, t=torch.int32), empty(3, t=torch.int32), empty(3, t=torch.int64)
    k, role, idx = empty(0, 2, d, t=torch.bfloat16), empty(0), empty(0, t=torch.int32)
    for q4 in (False, True):
        n, status = torch.full((3,), 9, dtype=torch.int32, device="cuda"), empty(1, t=torch.int32)
        if q4:
            codes, scales = empty(0, 2, d // 2), empty(0, 2, d // 32)
            st = sonic.kv_compact_q4(cu, role, k, k, codes, scales, codes, scales, off, cap, n, idx, status, 0)
        else:
            st = sonic.kv_compact(cu, role, k, k, k, k, off, cap, n, idx, status, 0)
        assert st == sonic.OK, (q4, sonic.status_string(st))
        assert n.tolist() == [0, 0, 0] and int(status.item()) == 0
