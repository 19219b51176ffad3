"""Pins of the 4-bit row and eviction oracles."""
import numpy as np
import pytest

import workloads as W
from oracle import decode as OD
from oracle import evict as OE
from oracle import q4 as OQ
from oracle.attention import bf16_bits_to_f64


def bits(x):
    return W.f32_to_bf16_bits(np.asarray(x, np.float32))


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.03125, 1), (3.5, -1), (3.515625, 0), (6.0, 0), (1.0, -2), (0.875, -3), (0.0, -127),
                                   (2.0 ** -126, -127), (3.3e38, 125), (2.0 ** 127, 125)])
def test_scale_is_the_smallest_power_that_fits(top, e):
    block = np.zeros(32)
    block[5] = -top
    _, scale = OQ.encode(bits(block))
    assert int(scale[0]) - 127 == e


def test_values_go_to_the_nearest_number_ties_to_the_even_index():
    x = [0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 1.74, 2.5, 2.52, 3.5, 3.48, 5.0, 5.03, 6.9, 6.0, -0.25, -0.75, -5.0, -0.0]
    want = [0, .5, 1, .5, 1, 1.5, 2, 1.5, 2, 3, 4, 3, 4, 6, 6, 6, 0, -1, -4, 0]
    block = np.zeros(32)
    block[:len(x)] = x
    block[31] = 7.0
    assert np.array_equal(OQ.rounded(bits(block))[:len(x)], want)


def test_a_block_with_infinity_or_nan_is_nan_and_its_neighbours_are_not():
    b = bits(np.ones((3, 64)))
    b[0, 40], b[1, 3] = 0x7F80, 0x7FC1
    nan = np.isnan(OQ.rounded(b))
    assert nan[0, 32:].all() and not nan[0, :32].any() and nan[1, :32].all() and not nan[1, 32:].any() and not nan[2].any()


def test_rounding_error_bound_and_rounding_again_changes_nothing():
    rng = np.random.default_rng(3)
    x = bits(rng.standard_normal((200, 64)) * np.exp(4 * rng.standard_normal((200, 1))))
    v, f = OQ.rounded(x), bf16_bits_to_f64(x)
    _, scale = OQ.encode(x)
    step = np.repeat(np.ldexp(1.0, scale.astype(int) - 127), 32, axis=-1)
    assert np.all(np.abs(v - f) <= np.maximum(step / 4, np.abs(f) / 5))
    assert np.array_equal(bf16_bits_to_f64(bits(v)), v)           # bf16 holds every value
    again = OQ.encode(bits(v))
    assert np.array_equal(OQ.decode(*again), v)
    assert np.array_equal(OQ.unpack(OQ.pack(again[0])), again[0])


def test_attention_and_weights_agree_with_the_decode_oracle():
    rng = np.random.default_rng(4)
    q, k, v = (bits(rng.standard_normal(s)) for s in ((6, 64), (19, 2, 64), (19, 2, 64)))
    out, w = OE.attend(q, bf16_bits_to_f64(k), bf16_bits_to_f64(v))
    assert np.allclose(out, OD.decode_step(q, k[:-1], v[:-1], k[-1], v[-1]), atol=1e-12)
    assert abs(w.sum() - 1) < 1e-12


@pytest.mark.parametrize("weight,head,tail,budget,want", [
    ([5, 1, 4, 2, 3], 0, 0, 3, [0, 2, 4]),
    ([5, 1, 4, 2, 3], 0, 0, 5, [0, 1, 2, 3, 4]),
    ([5, 1, 4, 2, 3], 2, 1, 4, [0, 1, 2, 4]),
    ([5, 1, 4, 2, 3], 2, 2, 1, [0, 1, 3, 4]),
    ([5, 1, 4, 2, 3], 9, 9, 0, [0, 1, 2, 3, 4]),
    ([1, 1, 1, 1], 0, 0, 2, [0, 1]),
    ([0.0, -0.0, np.nan, -np.inf], 0, 0, 3, [0, 1, 2]),
    ([np.nan, -np.inf, -1.0], 0, 0, 2, [0, 2]),
    ([], 1, 1, 0, []),
])
def test_kept_rows(weight, head, tail, budget, want):
    assert OE.kept_rows(np.array(weight, float), head, tail, budget).tolist() == want
