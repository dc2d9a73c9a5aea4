"""The oracle's 8-bit cache at the top of the float32 range."""
import numpy as np

from oracle import cache as oc


def test_largest_numbers_stay_finite():
    """256 2^120 is no float32: what would round to it is kept as 240 2^120, and half a step is still the bound."""
    x = np.zeros((6, 64))
    x[:, 0] = [2.0 ** 128 - 2.0 ** 104, 248 * 2.0 ** 120, 247.9 * 2.0 ** 120, 449 * 2.0 ** 119, 448 * 2.0 ** 119, -3.4e38]
    x[:, 1] = 2.0 ** 126
    y, e = oc.quantise(x)
    assert e.tolist() == [120, 120, 120, 120, 119, 120]
    assert np.isfinite(y.astype(np.float32)).all() and np.abs(y).max() == 240 * 2.0 ** 120
    assert (np.abs(y - x) <= 2.0 ** -4 * np.abs(x)).all()
    again, e2 = oc.quantise(y)
    assert np.array_equal(again, y)
