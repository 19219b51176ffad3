"""Attention of drafted tokens with 32-bit outputs on inputs whose scores are exact, so that what the probabilities are made
of shows in the outputs: a bar that a probability in two bf16 parts would not pass.

Every column sees two rows that count, with scores 0 and -x (0.05 <= x <= 1 in log2 units) and values 0 and 1 or 1 and 0;
all others' exact weights are below 2^-4000, 0 in 32 bits.  With p = 2^-x the outputs are p / (1 + p) and 1 / (1 + p).

Bar, with U = 2^-24, half a step of fp32.  The factor of the scores is rounded twice and the exponent once: off by 3 U at most,
and p by 3 ln 2 U < 2.1 U of itself; the hardware's exponential by 2^-22 = 4 U; three bf16 parts leave 2^-26 = U / 4 of p.  So
p is off by 6.4 U of itself, and either output by p / (1 + p)^2 <= 1/4 of that: 1.6 U.  The sums of p's parts and of 1 are
exact up to the last part (8 and 16 bits), whose addition may be cut off: 2 U of the sum above and of that below, U for the
inverse and U for the product, 6 U of an output below 2/3: 4 U.  Together 5.6 U; the bar is 8 U.
A p in two parts is off by up to 2^-18, the outputs by up to 2^-18 / (1 + p)^2: 16 to 28 U.
"""
import numpy as np
import pytest

import workloads as W
from oracle.attention import bf16_bits_to_f64
from paper_2601_21927_amd import sonic
from tests import gpu_helpers as H
from tests.test_gpu_decode_exact import set_rows
from tests.test_gpu_q4 import Cache
from tests.test_gpu_tree import Step

pytestmark = pytest.mark.gpu

BAR = 8 * 2.0 ** -24


def bits(x):
    return W.f32_to_bf16_bits(np.asarray(x, np.float32))


def rounded(x):
    return bf16_bits_to_f64(bits(x))


def pairs(rng, B, lens, Hq, Hkv, d, nodes, q4):
    """Even requests have their two rows in one block of the cache, odd ones among their nodes (stars: the root, and each node's
    own).  Channel 0 carries the rows that do not count, channel 1 the scores."""
    c = Cache(rng, lens, 1, Hkv, d, q4)
    s = Step(rng, c, Hq, nodes, "star")
    k, v = (np.zeros_like(x) for x in c.bits)
    kn, vn = np.zeros_like(s.k), np.zeros_like(s.v)
    k[..., 0] = kn[..., 0] = bits(-6.0)

    def put(keys, values, at, second):
        keys[at, :, 0], keys[at, :, 1] = 0, bits(-1.0 if second else 0.0)
        values[at, :, (0 if second else 1)::2] = bits(1.0)
    for b, n in enumerate(lens):
        if b % 2 == 0:
            block = 32 * int(rng.integers(0, (n - 2) // 32 + 1))
            first, second = block + rng.permutation(min(32, n - block))[:2]
            put(k, v, int(c.off[b]) + first, False)
            put(k, v, int(c.off[b]) + second, True)
        elif nodes[b]:
            put(kn, vn, s.cu[b], False)
            for i in range(1, nodes[b]):
                put(kn, vn, s.cu[b] + i, True)
    set_rows(c, k, v)
    s.q[...], s.k[...], s.v[...] = 0, kn, vn
    s.q[..., 0] = bits(4096.0)
    x = rng.uniform(0.05, 1.0, s.q.shape[:2])
    s.q[..., 1] = bits(x * np.sqrt(d) / np.log2(np.e))
    return c, s


def two_parts(q1, d):
    """How far outputs are off whose p are in two bf16 parts, at most."""
    p = np.exp2(-q1 / np.sqrt(d) * np.log2(np.e))
    high = rounded(p)
    some = high + rounded(p - high)
    return max(np.abs(some / (1 + some) - p / (1 + p)).max(), np.abs(1 / (1 + some) - 1 / (1 + p)).max())


SHAPES = [([70, 0, 400, 33], 4, 2, 64, [5, 30, 3, 33]), ([1328, 40] * 4, 32, 8, 128, [32, 9] * 4), ([40], 28, 4, 128, [20]),
          ([9000, 100], 8, 2, 128, [9, 4]), ([20000], 4, 1, 64, [7]), ([3, 2, 17, 5], 7, 1, 128, [2, 30, 1, 4])]


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,d,nodes", SHAPES)
def test_two_rows(lens, Hq, Hkv, d, nodes, q4):
    H.need_gpu()
    c, s = pairs(np.random.default_rng(sum(lens) + Hq), len(lens), lens, Hq, Hkv, d, nodes, q4)
    check(s)


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [17, 33])
@pytest.mark.parametrize("most", [8, 16, 32, 64, 68])
def test_two_rows_in_every_cut(B, d, q4, most):
    """136 and 264 (request, kv-head) pairs with up to 16 to 136 rows a kv-head: tiles of every size."""
    H.need_gpu()
    rng = np.random.default_rng(B + d + most)
    lens, nodes = [int(x) for x in rng.integers(2, 70, B)], [int(x) for x in rng.integers(0, 4, B)]
    lens[4], nodes[4], nodes[5] = 3300, most // 2 + 1, most
    c, s = pairs(rng, B, lens, 16, 8, d, nodes, q4)
    check(s)


def check(s):
    got = s.run("fp32")
    assert int(s.status.item()) == sonic.OK
    assert two_parts(bf16_bits_to_f64(s.q[..., 1]), s.c.d) > 1.5 * BAR
    for b in range(len(s.nodes)):
        if s.nodes[b]:
            want, top = s.expect(b)
            mine = got[s.cu[b]:s.cu[b + 1]]
            assert top == 1.0 and 0.2 < want.max() <= 1.0
            assert np.abs(mine - want).max() <= BAR, (b, np.abs(mine - want).max() / BAR)
