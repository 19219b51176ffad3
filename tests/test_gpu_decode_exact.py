"""Decode steps on inputs whose scores are exact, so that what the probabilities are made of shows in the outputs."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import evict as OE
from oracle import q4 as OQ
from oracle.attention import bf16_bits_to_f64
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import bf16_to_device
from tests import gpu_helpers as H
from tests.test_gpu_q4 import EPS, Cache, i32, normal_bits

pytestmark = pytest.mark.gpu


def set_rows(c, k_bits, v_bits):
    """All rows of a Cache anew."""
    c.bits = [k_bits, v_bits]
    c.values = [OQ.rounded(x) if c.q4 else bf16_bits_to_f64(x) for x in c.bits]
    d = c.dev
    if c.q4:
        for x, codes, scales in ((k_bits, d.k, d.k_scale), (v_bits, d.v, d.v_scale)):
            a, s = OQ.encode(x)
            codes.copy_(torch.from_numpy(OQ.pack(a)))
            scales.copy_(torch.from_numpy(s))
    else:
        d.k.copy_(bf16_to_device(k_bits))
        d.v.copy_(bf16_to_device(v_bits))


def decode(c, q, k, v, weighted=True, max_ctx=None):
    out = torch.full((len(c.lens),) + q.shape[1:], 7.0, device="cuda")
    args = (bf16_to_device(q), bf16_to_device(k), bf16_to_device(v), out, c.status, max_ctx or c.max_ctx)
    st = c.dev.decode(*args, weighted=weighted) if c.q4 else (c.dev.decode_weighted if weighted else c.dev.decode)(*args)
    assert st == sonic.OK and int(c.status.item()) == 0
    return out.cpu().numpy()


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,lens,first", [(4, 2, 64, [70, 400, 33], 64), (8, 1, 128, [100, 1500], 96), (6, 1, 64, [4000, 90], 640),
                                                 (8, 8, 64, [2100] + [90] * 39, 64)])
def test_scores_that_pass_the_range_below_weigh_nothing(Hq, Hkv, d, lens, first, q4):
    """The first rows' scores are -infinity in 32 bits, whole blocks of them: weight 0, as their exact scores have."""
    H.need_gpu()
    rng = np.random.default_rng(41 + Hq + q4)
    c = Cache(rng, lens, 2, Hkv, d, q4)
    k, v = c.bits
    k[..., :32] = 0
    for o, n in zip(c.off, lens):
        k[o:o + min(first, n), :, 0] = W.f32_to_bf16_bits(np.float32([-6.0]))[0]
        k[o + 3:o + n:50, :, 0] = 0xC0C0   # -6 again, and alone among rows of 0
        k[o + n - 1, :, 0] = 0
    set_rows(c, k, v)
    B = len(lens)
    q, kn, vn = (normal_bits(rng, B, h, d) for h in (Hq, Hkv, Hkv))
    q[..., 0] = W.f32_to_bf16_bits(np.float32([3e38]))[0]
    kn[..., :32] = 0
    out = decode(c, q, kn, vn)
    assert np.isfinite(out).all()
    c.check(q, kn, vn, out)
