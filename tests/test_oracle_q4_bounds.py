"""The error bound that the header states for 4-bit rows, at the ends of the bf16 range."""
import numpy as np
import pytest

from oracle import q4 as OQ
from oracle.attention import bf16_bits_to_f64


@pytest.mark.parametrize("lowest,highest", [(0x0000, 0x0800), (0x3F00, 0x4100), (0x7E00, 0x7F80)])
def test_error_bound_over_whole_ranges_of_magnitudes(lowest, highest):
    """Every finite pattern of a range as a block's largest, over fractions of itself and the smallest numbers."""
    top = np.arange(lowest, highest, dtype=np.uint16)
    rng = np.random.default_rng(1)
    below = (top[:, None] * rng.random((len(top), 31)) ** 0.05).astype(np.uint16)   # mostly within a few powers of two
    below[:, ::7] = rng.integers(0, 3, size=below[:, ::7].shape)
    block = np.concatenate([top[:, None], below | (rng.integers(0, 2, size=below.shape) << 15).astype(np.uint16)], 1)
    x, v = bf16_bits_to_f64(block), OQ.rounded(block)
    a = np.abs(x).max(1)
    e = OQ.encode(block)[1][:, 0].astype(int) - 127
    step = np.ldexp(1.0, e)
    limit = np.ldexp(7.0, 125)
    err, bound = np.abs(v - x), np.maximum(step[:, None] / 4, np.abs(x) / 5)
    over = np.abs(x) > limit
    assert np.all(err[~over] <= bound[~over])
    assert np.all(err[over] < np.abs(x[over]) / 4) and np.all(np.abs(v[over]) == np.ldexp(6.0, 125))
    plain = (e > -127) & (a <= limit)
    assert np.all((step[plain] >= a[plain] / 7) & (step[plain] < 2 * a[plain] / 7))
    assert np.array_equal(e == -127, a <= np.ldexp(7.0, -127)) and np.all(e[a > limit] == 125)
    if lowest == 0:
        assert (e == -127).sum() > 100 and (e[(e == -127) & (a < np.ldexp(7.0, -128))].size > 50)
    if highest == 0x7F80:
        assert over.sum() > 31
