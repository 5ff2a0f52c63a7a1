"""The 64-bit form of the 8-bit moments for millions of elements is the plain one."""
import numpy as np
import pytest

from tests import fullrank_reference as ref


@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("n", [1, 127, 128, 129, 1000])
def test_all_blocks_at_once(signed, n):
    rng = np.random.default_rng(n)
    x = rng.standard_normal(n) * 2.0 ** rng.integers(-40, 3, n)
    x[rng.random(n) < 0.2] = 0
    x[:1] *= 2.0 ** -135                       # (a block of one value that fp32 holds as a subnormal)
    if not signed:
        x = np.abs(x)
    if n == 1000:
        x[:128] = 0
        x[130], x[300], x[600] = np.inf, 2.0 ** 127 * 1.5, 2.0 ** -3
        x[512:640] = np.where(np.arange(128) == 88, 2.0 ** -3, x[512:640] * 2.0 ** -6)
    w = rng.integers(0, 1 << 17, n)
    with np.errstate(invalid="ignore"):
        a, b = ref.in_8_bits(x, w, signed), ref.in_8_bits_of_many(x, w, signed)
    assert np.array_equal(a, b, equal_nan=True)
