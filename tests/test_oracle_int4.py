"""Pins of the 4-bit row format."""
import numpy as np

from oracle import int4


def test_hand_worked_row():
    x = np.array([7.0, -7.0, 3.4, -3.6, 0.5, 1.5, -2.5, 0.0])
    codes, s = int4.quantise_rows(x[None], np.ones(8))
    assert s[0] == 1.0
    np.testing.assert_array_equal(codes[0], [15, 1, 11, 4, 8, 10, 6, 8])          # ties go to the even integer
    np.testing.assert_array_equal(int4.values(codes, s, np.ones(8))[0], [7, -7, 3, -4, 0, 2, -2, 0])


def test_pack_round_trip_and_byte_order():
    rng = np.random.default_rng(0)
    c = rng.integers(1, 16, (5, 128)).astype(np.uint8)
    np.testing.assert_array_equal(int4.unpack(int4.pack(c)), c)
    assert int4.pack(np.array([[3, 14]], dtype=np.uint8))[0, 0] == 0xE3


def test_half_step_error_and_the_largest_element_exact():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(200, 128)).astype(np.float32)
    chan = np.exp(rng.normal(size=128)).astype(np.float32)
    x = (x * chan).astype(np.float32)
    codes, s = int4.quantise_rows(x, np.float32(1) / chan)
    v = int4.values(codes, s, chan)
    step = s[:, None].astype(np.float64) * chan
    assert (np.abs(v - x) <= step * (0.5 + 1e-5)).all()
    top = np.abs(x / chan).argmax(axis=1)
    got, ref = v[np.arange(200), top], x[np.arange(200), top]
    np.testing.assert_allclose(got, ref, rtol=1e-6)
    assert codes.min() >= 1 and codes.max() <= 15


def test_zero_rows_and_tiny_rows():
    codes, s = int4.quantise_rows(np.zeros((2, 8)), np.ones(8))
    assert (codes == 8).all() and (s == 0).all()
    codes, s = int4.quantise_rows(np.full((1, 8), 1e-38, dtype=np.float32), np.ones(8))
    assert (codes == 15).all() and s[0] > 0
