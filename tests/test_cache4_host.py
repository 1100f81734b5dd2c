"""The 4-bit form's restatement against its definition, and the refusals of its
entry points that need no GPU."""

import numpy as np

from oracle import cache4_oracle as O4


def test_four_significant_bits_rounded_up():
    t = np.array([0.0, 1.0, 15.0, 15.5, 17.0, 0.3, 2.0 ** -20, 1.0000001, 61440.0, 61441.0], np.float32)
    want = np.array([0.0, 1.0, 15.0, 16.0, 18.0, 0.3125, 2.0 ** -20, 1.125, 61440.0, 65536.0], np.float32)
    np.testing.assert_array_equal(O4.four_bits_up(t), want)
    rng = np.random.default_rng(0)
    x = np.exp(rng.uniform(-30, 30, 10000)).astype(np.float32)
    y = O4.four_bits_up(x)
    m, _ = np.frexp(y)
    assert (m * 16 == np.rint(m * 16)).all() and (y >= x).all() and (y <= x * 1.125).all()


def test_held_values_are_near_and_exact_in_bf16():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((50, 128)) * np.exp(rng.uniform(-3, 3, (50, 1)))).astype(np.float32)
    code, step = O4.quantise(x)
    assert code.min() >= 0 and code.max() <= 15
    held = O4.values(code, step)
    # half a step from the nearest whole number of steps (the largest value at 7.5 steps included)
    assert (np.abs(held - x) <= 0.5 * np.repeat(step, 32, -1) * (1 + 2.0 ** -20)).all()
    bits = held.astype(np.float32).view(np.uint32)
    assert not (bits & 0xFFFF).any()
    np.testing.assert_array_equal(O4.unpack(O4.pack(code)), code)
    assert (O4.pack(code)[:, 0] & 15 == code[:, 0]).all()


def test_rotation_keeps_lengths():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 64))
    a = rng.uniform(0, 6, (3, 16))
    for pairs in (False, True):
        y = O4.rotate(x, np.cos(a), np.sin(a), pairs, np.float64)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        np.testing.assert_array_equal(y[:, 32:], x[:, 32:])
        back = O4.rotate(y, np.cos(a), -np.sin(a), pairs, np.float64)
        np.testing.assert_allclose(back, x, atol=1e-12)


def test_refusals_without_a_context(lib):
    none = lib.VP_ERR_NOT_INITIALIZED
    assert lib.lib.vp_append(None, 1, 1, *([None] * 10)) == none
    assert lib.lib.vp_append4(None, 1, 1, *([None] * 12)) == none
    assert lib.lib.vp_reserve4(None, 1) == none
    assert lib.lib.vp_attend4(None, 1, 1, *([None] * 9)) == none
