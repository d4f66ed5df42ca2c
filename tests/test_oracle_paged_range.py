"""The paged cache's oracle at the top of float32's range (CPU only)."""
import numpy as np
import pytest

from oracle import paged as ref

F32_MAX = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("fmt,step,top,code", [("e4m3", 16 * 2.0 ** 120, 240 * 2.0 ** 120, 247),
                                               ("int8", 2.0 ** 122, 63 * 2.0 ** 122, 249)])
def test_largest_finite_rows_stay_finite(fmt, step, top, code):
    """Values that would be rounded to 2^128 take the number before it, at most
    a step away; the others are off by half a step at most, as everywhere."""
    rng = np.random.default_rng(0)
    x = rng.uniform(-1, 1, (500, 64)) * 2.0 ** 128
    x[:, 0] = F32_MAX * rng.choice([-1, 1], 500)
    x[0, 1:5] = [255 * 2.0 ** 120, 1.9375 * 2.0 ** 127, 1.96875 * 2.0 ** 127, 1.984375 * 2.0 ** 127]
    x = x.astype(np.float32).astype(np.float64)
    q, c = ref.quantise(x, fmt)
    v = ref.value(q, c)
    assert (c == code).all() and np.abs(v).max() == top
    far = np.abs(x) >= top + step / 2
    assert far.any() and (v[far] == np.sign(x[far]) * top).all() and (np.abs(v - x)[far] < step).all()
    assert (np.abs(v - x)[~far] <= step / 2).all()


@pytest.mark.parametrize("fmt,border", [("e4m3", 1.75 * 2.0 ** 127), ("int8", 1.984375 * 2.0 ** 127)])
def test_rows_of_the_exponent_below_are_as_they_were(fmt, border):
    q, c = ref.quantise(np.array([[border, -border, 2.0 ** 126]]), fmt)
    assert ref.value(q, c)[0, :2].tolist() == [border, -border] and np.abs(q).max() == ref.LIMIT[fmt]
