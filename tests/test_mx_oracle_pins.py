"""The oracle of the microscaled 4-bit format against values worked out by hand and against a search over all codes."""
import numpy as np
import pytest

from oracle import mx_oracle as mx


def one_block(values):
    v = np.zeros((1, 32))
    v[0, :len(values)] = values
    return v


def test_codes_of_the_grid_and_of_its_borders():
    """the largest entry 6 makes the scale 1: floor(log2 6) - 2 = 0"""
    v = [6.0, 0.0, -0.0, 0.5, -1.5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, 0.2500001, 4.9999999, 5.0000001]
    code, scale = mx.quantize(one_block(v))
    assert scale[0, 0] == 127 and (scale[0, 1:] == 0).all() and scale.shape == (1, 4)
    assert list(code[0, :16]) == [7, 0, 8, 1, 11, 0, 2, 2, 4, 4, 6, 6, 14, 1, 6, 7]
    assert (code[0, 16:] == 0).all()
    assert mx.pack(code)[0, :3].tolist() == [0x07, 0x18, 0x0B]


@pytest.mark.parametrize("top,byte,code", [(7.999, 127, 7), (8.0, 128, 6), (4.0, 127, 6), (3.9999, 126, 7), (2.0 ** -126, 0, 4), (2.0 ** -149, 0, 0), (2.0 ** 127 * 1.5, 252, 7),
                                           (65504.0, 140, 7), (2.0 ** -24, 101, 6), (0.0, 0, 0)])
def test_scale_of_a_block(top, byte, code):
    c, s = mx.quantize(one_block([-top]))
    assert s[0, 0] == byte and c[0, 0] & 7 == code


def test_blocks_that_hold_no_number():
    for bad in (np.inf, -np.inf, np.nan):
        v = np.concatenate([one_block([1.0, bad, 3.0]), one_block([1.0])], axis=1)
        c, s = mx.quantize(v)
        assert s[0].tolist() == [255, 125, 0, 0] and (c[0, :32] == 0).all()
        assert np.isnan(mx.expand(mx.pack(c), s, 64)[0, :32]).all() and mx.expand(mx.pack(c), s, 64)[0, 32] == 1.0


def test_every_element_gets_a_nearest_value():
    rng = np.random.default_rng(5)
    v = rng.standard_t(4, (40, 96)) * np.exp(rng.normal(size=(40, 1)) * 10)
    c, s = mx.quantize(v)
    back = mx.expand(mx.pack(c), s, 96)
    scale = np.ldexp(1.0, s.astype(int) - 127)[:, :3].repeat(32, axis=1)
    all_values = mx.GRID[None, None, :] * scale[:, :, None]
    nearest = np.abs(np.abs(v)[:, :, None] - all_values).min(axis=2)
    assert np.array_equal(np.abs(np.abs(v) - np.abs(back)), nearest)
    assert (np.sign(back) * np.sign(v) >= 0).all()
    top = np.abs(v).reshape(40, 3, 32).max(axis=2) / scale[:, ::32]
    assert (top >= 4).all() and (top < 8).all()


def test_types():
    v = np.array([1.0, -2.5, 65504.0, 2.0 ** -24, 3.0])
    for kind in ("f16", "f32"):
        assert np.array_equal(mx.to_double(mx.from_double(v, kind), kind), v)
    assert mx.from_double(np.array([1.0, 1.00390625, 1.01171875, -3.0]), "bf16").tolist() == [0x3F80, 0x3F80, 0x3F82, 0xC040]
