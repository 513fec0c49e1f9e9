"""The binding's rounding of uniform numbers to fp32."""
import numpy as np

from paper_2608_10139_gb300 import aiq


def test_numbers_below_1_stay_below_1():
    u = np.array([[0.0, 0.5, 1 - 2.0 ** -53, 1 - 2.0 ** -25], [1 - 2.0 ** -24, 0.999, 1.0, -0.1]])
    f = aiq._uniforms(u)
    assert f.dtype == np.float32 and f.shape == u.shape and f.flags.c_contiguous
    top = np.float32(1 - 2.0 ** -24)
    assert np.array_equal(f, np.array([[0, 0.5, top, top], [top, np.float32(0.999), 1, np.float32(-0.1)]], np.float32))


def test_32_bit_numbers_are_taken_as_they_are():
    u = np.random.default_rng(0).random((7, 5)).astype(np.float32)
    assert aiq._uniforms(u) is u
    assert np.array_equal(aiq._uniforms(u.T), u.T) and aiq._uniforms(u.T).flags.c_contiguous
    assert np.isnan(aiq._uniforms([[float("nan"), float("inf")]])[0, 0])


def test_the_order_in_memory_is_that_of_rows():
    u = np.asfortranarray(np.array([[0.25, 1 - 2.0 ** -53, 0.5], [0.125, 0.75, 1 - 2.0 ** -30]]))
    f = aiq._uniforms(u)
    assert f.flags.c_contiguous
    assert np.array_equal(np.frombuffer(f.tobytes(), np.float32), f.ravel())
    top = np.float32(1 - 2.0 ** -24)
    assert f.ravel().tolist() == [0.25, top, 0.5, 0.125, 0.75, top] and u[0, 1] == 1 - 2.0 ** -53
