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


U = 2.0 ** -24   # half a step of fp32, relative
HEADS = [(4, 2, 64), (8, 1, 64), (32, 8, 128), (28, 4, 128), (5, 1, 128), (6, 2, 64)]


def two_row_case(Hq, Hkv, d, q4, lens=(1, 34, 75, 333, 1500)):
    """Requests whose last row (score 0) and new row (score -x, 0.05 <= x <= 1 in log2 units) share everything: all other
    rows' probabilities are 0 in 32 bits and below 2^-4000 exactly.  All dot products are exact."""
    rng = np.random.default_rng(Hq * 100 + d + q4)
    c = Cache(rng, lens, 2, Hkv, d, q4)
    c.weight[:] = 0.0
    c.dev.row_weight.zero_()
    one = W.f32_to_bf16_bits(np.float32([1.0, -1.0, -6.0, 4096.0]))
    k, v = (np.zeros_like(x) for x in c.bits)
    v[...] = normal_bits(rng, *v.shape)
    kn, vn = (np.zeros((len(lens), Hkv, d), np.uint16) for _ in range(2))
    k[..., 1] = one[2]
    last = [int(o) + n - 1 for o, n in zip(c.off, lens)]
    k[last] = 0
    kn[..., 0] = one[1]
    # (last, new): 1 and -1, 1 and 1, 0 and 1, 1 and 0
    pairs = np.array([[one[0], one[1]], [one[0], one[0]], [0, one[0]], [one[0], 0]], np.uint16)
    v[last] = pairs[np.arange(d) % 4, 0]
    vn[...] = pairs[np.arange(d) % 4, 1]
    set_rows(c, k, v)
    q = np.zeros((len(lens), Hq, d), np.uint16)
    x = 0.05 + 0.95 * rng.random((len(lens), Hq))
    q[..., 0] = W.f32_to_bf16_bits((x * 0.999 * np.sqrt(d) / np.log2(np.e)).astype(np.float32))
    q[..., 1] = one[3]
    return c, q, kn, vn


def planted(c, b, q, wrong):
    """The two rows' output when a probability has two bf16 parts, or the sum of the probabilities leaves out the third."""
    bf16 = lambda x: torch.tensor(x, dtype=torch.float32).bfloat16().double().numpy()
    p = np.exp(-bf16_bits_to_f64(q[b, :, 0]) / np.sqrt(c.d))[:, None]
    parts = bf16(p)
    parts = parts + bf16(p - parts)
    top = parts if wrong == "two parts" else p
    va, vb = np.array([1, 1, 0, 1.0]), np.array([-1, 1, 1, 0.0])
    return (va + top * vb) / (1 + parts)


@pytest.mark.parametrize("q4,weighted", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_probabilities_go_in_whole(Hq, Hkv, d, q4, weighted):
    """In units of U = 2^-24, with values of at most 1.  A score x in log2 units is off by 3 |x| (the scale's two roundings,
    and its product's), its exponential by 2 (one unit in the last place, p >= 1/2) and the three bf16 parts by 1/4: p by
    2.1 + 2 + 0.25 of itself, which moves (a + p b) / (1 + p) by 2.2 at most.  Numerator and denominator are four addends
    each, with 2 for every addition (a unit in the last place): 8 and 8.  The quotient adds 1: 20 with what was rounded up.
    Two parts of p leave up to 2^-18, 64 units, which moves the output by up to 57; the third left out of the sum, 42.

    A weight is exp2(x - l): x off by 3, l = log2(1 + p) by (2.2 + 8) / ln 2 and 1, the difference by 1, so the weight by
    ln 2 * 19.7 = 13.7 of itself, its exponential by 2, its mean by one for each q-head and 2."""
    H.need_gpu()
    c, q, kn, vn = two_row_case(Hq, Hkv, d, q4)
    out = decode(c, q, kn, vn, weighted=weighted)
    got_w = c.dev.row_weight.cpu().numpy()
    seen = dict.fromkeys(("two parts", "sum of two"), 0.0)
    for b, (o, n) in enumerate(zip(c.off, c.lens)):
        want, w = c.expect(b, q, kn, vn)
        assert np.abs(out[b] - want).max() <= 20 * U, (b, np.abs(out[b] - want).max() / U)
        if weighted:
            assert np.all(np.abs(got_w[o:o + n + 1] - w) <= (18 + Hq) * U * w), b
        for wrong in seen:
            seen[wrong] = max(seen[wrong], np.abs(np.tile(planted(c, b, q, wrong), d // 4) - want).max())
    assert all(x > 25 * U for x in seen.values()), seen     # the bar tells these mistakes


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (16, 2, 128)])
def test_weights_of_large_scores(Hq, Hkv, d, q4):
    """Scores of several hundred.  With S the largest sum of |q k| over a row, scaled, in log2 units: a score is off by
    2 d U S (an addition for each product) and 3 U S for the scale, the normaliser by as much and by 2 U for each
    row of its sum and 16 U for the probabilities' own errors, their difference by 2 U S; then the exponential and the mean
    as above."""
    H.need_gpu()
    rng = np.random.default_rng(71 + q4 + d)
    c = Cache(rng, [500, 3, 47], 2, Hkv, d, q4)
    q, k, v, out = c.step(rng, Hq, scale=50.0)
    got = c.dev.row_weight.cpu().numpy()
    for b in range(3):
        o, n = int(c.off[b]), int(c.lens[b])
        _, w = c.expect(b, q, k, v)
        keys = np.abs(c.values[0][o:o + n + 1])
        S = max((keys[:, h * Hkv // Hq] @ np.abs(bf16_bits_to_f64(q[b, h]))).max() for h in range(Hq)) * np.log2(np.e) / np.sqrt(d)
        rel = np.exp2((2 * (2 * d + 3) + 2) * U * S + (2 * n + 16) * U) - 1 + (18 + Hq) * U
        assert rel < 0.1
        full = w + np.concatenate([c.weight[o:o + n].astype(np.float64), [0.0]])
        assert np.all(np.abs(got[o:o + n + 1] - full) <= rel * w + U * full + 2.0 ** -126), b
