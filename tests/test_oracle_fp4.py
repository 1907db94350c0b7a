"""The oracle of a cache in 4 bits against cases worked by hand and the format's own identities."""
import numpy as np
import pytest

from oracle import worker as ow


def test_codes_by_hand():
    x = np.zeros(40)
    x[:12] = 7, -6, 5, 4.5, 3.5, 2.5, 1.75, 1.25, 0.75, -0.25, 0.26, -0.0
    x[32:35] = 7.25, 14, -3
    codes, scales = ow.fp4_encode(x, "bf16")
    assert codes.shape == (32,) and scales.tolist() == [127, 128]
    # 7 -> 6, -6, 5 -> 4 (even), 4.5 -> 4, 3.5 -> 4, 2.5 -> 2, 1.75 -> 2, 1.25 -> 1, 0.75 -> 1, -0.25 -> -0, 0.26 -> 0.5, -0
    assert codes[:6].tolist() == [0x7 | 0xf0, 0x6 | 0x60, 0x6 | 0x40, 0x4 | 0x20, 0x2 | 0x80, 0x1 | 0x80]
    # in steps of 2: 3.625 -> 4, 7 -> 6, -1.5
    assert codes[16:18].tolist() == [0x6 | 0x70, 0xb] and not codes[18:].any()
    y = ow.fp4_decode(codes, scales, 40)
    assert y[:12].tolist() == [6, -6, 4, 4, 4, 2, 2, 1, 1, 0, 0.5, 0] and y[32:36].tolist() == [8, 12, -3, 0]


def test_ends_of_the_range_by_hand():
    for dtype, lo, hi in (("bf16", -125, 125), ("fp16", -23, 13)):
        x = np.zeros((5, 32))
        x[0, 0], x[1, 0], x[2, 0], x[3, 3] = 7 * 2.0 ** hi, 8 * 2.0 ** hi, 0.25 * 2.0 ** lo, 2.0 ** lo
        codes, scales = ow.fp4_encode(x, dtype)
        assert scales[:, 0].tolist() == [hi + 127, hi + 127, lo + 127, lo + 127, lo + 127]
        y = ow.fp4_decode(codes, scales, 32)
        assert y[0, 0] == y[1, 0] == 6 * 2.0 ** hi and not y[2].any() and y[3, 3] == 2.0 ** lo and not y[4].any()
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones((1, 64))
        x[0, 40] = bad
        codes, scales = ow.fp4_encode(x, "bf16")
        assert scales[0, 1] == 255 and not codes[0, 16:].any()
        y = ow.fp4_decode(codes, scales, 64)
        assert (y[0, :32] == 1).all() and np.isnan(y[0, 32:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_held_are_near_and_stay(dtype):
    rng = np.random.default_rng(4)
    x = rng.normal(size=(200, 72)) * 2.0 ** rng.integers(-9, 9, (200, 1))
    codes, scales = ow.fp4_encode(x, dtype)
    y = ow.fp4_decode(codes, scales, 72)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)[:, :72]
    m = np.abs(x) / step
    assert (np.abs(x - y) <= step * np.where(m < 2, 0.25, np.where(m < 4, 0.5, 1.0))).all() and (m <= 7).all()
    # what is held is held again as it is
    again = ow.fp4_encode(y, dtype)
    assert np.array_equal(ow.fp4_decode(*again, 72), y)
