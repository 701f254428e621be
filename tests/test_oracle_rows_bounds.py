"""The stated errors of the 8-bit form over the whole range of exponents, on the oracle."""
import numpy as np

from oracle import rows as R


def test_error_by_exponent():
    r = np.random.default_rng(5)
    at = np.arange(-148, 128)                                  # every power of two of a float32
    x = (r.uniform(-1, 1, (at.size, 40, 32)) * 2.0 ** at[:, None, None]).astype(np.float32).astype(np.float64)
    x[:, 0, 0] = (2 - 2.0 ** -23) * 2.0 ** at                  # up to the largest finite value
    codes, scales = R.encode(x.reshape(-1))
    err = np.abs(R.decode(codes, scales).reshape(x.shape) - x).max(-1).reshape(-1)
    top, s = np.abs(x).max(-1).reshape(-1), scales.astype(np.int64)
    half = 2.0 ** (s - 134.0)
    low, high, mid = s == 7, s == 254, (s > 7) & (s < 254)
    assert low.any() and high.any() and mid.any()
    assert np.all(err[mid] <= half[mid]) and np.all(half[mid] <= top[mid] / 127)
    assert np.all(err[low] <= 2.0 ** -127) and np.any(err[low] > top[low] / 127)
    assert np.all(err[high] < 2 * half[high]) and np.any(err[high] > half[high])
