"""What the 8-bit cache's row format promises, from its definition in 64 bits (CPU)."""

import numpy as np
import pytest

import _kv8 as R


def _rows(seed, n=4000, D=64):
    g = np.random.default_rng([20397, 90, seed])
    x = g.standard_normal((n, D)) * np.exp2(g.integers(-60, 60, (n, 1)) + g.random((n, 1)))
    x[::3] *= np.exp2(-g.integers(0, 24, (len(x[::3]), D)).astype(np.float64))    # elements far below their row's largest
    return x


def test_values_quantised_again_are_the_same_and_bytes_move_once():
    """The largest code of a row with amax in (224, 232] 2^e is 224 = 448 / 2: its second byte is one less.  No
    other row's bytes move, and none moves twice."""
    x = _rows(1)
    x[:3, 0] = [232.0, -225.0, 224.001]                    # borders of the rows that move (232: a tie, down)
    x[3:6, 0] = [224.0, 232.0001, -448.0]                  # and of those that do not
    x[:6, 1:] = np.clip(x[:6, 1:], -100, 100)
    val, byte = R.quantise(x)
    again, byte2 = R.quantise(val)
    third, byte3 = R.quantise(again)
    assert np.array_equal(val, again) and np.array_equal(val, third) and np.array_equal(byte2, byte3)
    y = np.abs(x).max(-1) / 2.0 ** (byte - 127.0)
    moved = (y > 224) & (y <= 232) & (byte > 27)
    assert moved[:3].all() and not moved[3:6].any() and 0.02 < moved.mean() < 0.1
    assert np.array_equal(byte2, byte - moved)


def _bounds_hold(x, got, rel, rel_from, below):
    """Off by at most `rel` of an element down to rel_from of its row's largest, by `below` of that under it."""
    amax = np.abs(x).max(-1, keepdims=True)
    err = np.abs(got - x)
    near = np.abs(x) >= rel_from * amax
    return np.all(err[near] <= rel * np.abs(x)[near]) and np.all((err <= below * amax)[~near])


def test_error_bounds():
    """Half a step of three mantissa bits in the normal codes' range, which begins below 2^-13.8 of a row's largest
    element, and half a subnormal step under it."""
    x = np.concatenate([_rows(2), _rows(3) * 2.0 ** 50])
    x[:5, 0] = 225.0                                     # the step is largest against amax just past 224
    x[:5, 1:] = np.clip(x[:5, 1:], -200, 200)
    x[:5, 1] = [7.5 * 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -6, 2.0 ** -6 * 1.0625]
    val, byte = R.quantise(x)
    e = byte[:, None] - 127.0
    assert np.all(np.abs(val - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (e - 10)))
    assert _bounds_hold(x, val, 2.0 ** -4, 2.0 ** -13.8, 2.0 ** -17.8)
    # neither holds further down
    assert not _bounds_hold(x, val, 2.0 ** -4, 2.0 ** -14, 2.0 ** -17.8)
    assert not _bounds_hold(x, val, 2.0 ** -4, 2.0 ** -13.8, 2.0 ** -18)


@pytest.mark.parametrize("amax", [2.0 ** -92, 1.01 * 2.0 ** -92.19, 2.0 ** -93, 2.0 ** -101, 2.0 ** -108])
def test_small_rows_have_the_step_of_the_least_exponent(amax):
    x = np.concatenate([np.linspace(-amax, amax, 999), [2.0 ** -110, -(2.0 ** -110), 1.0001 * 2.0 ** -110]])[None]
    val, byte = R.quantise(x)
    assert byte == 27
    assert np.all(np.abs(val - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -110))
    assert np.array_equal(val == 0, np.abs(x) <= 2.0 ** -110)


def test_rows_past_the_largest_value_are_held_to_it():
    top = 448 * 2.0 ** 119
    x = np.array([[top, 1.1 * top, -1.14 * top, 0.5 * top]])
    val, byte = R.quantise(x)
    assert byte == 246 and np.array_equal(val, [[top, top, -top, 0.5 * top]])


def test_a_query_in_two_terms():
    """hi is the query's code and lo that of 16 times the rest: exact for a bf16 of the normal codes' range, half a
    sixteenth of the subnormal step below it."""
    x = _rows(4)
    x[:4, 0] = 225.0
    x[:4, 1:] = np.clip(x[:4, 1:], -200, 200)
    x[:4, 1] = [2.0 ** -14, 3 * 2.0 ** -14, 2.0 ** -6 * (1 + 2.0 ** -7), 255 * 2.0 ** -14]
    b = 2.0 ** (np.floor(np.log2(np.abs(x))) - 7)
    x = np.rint(x / b) * b                               # bf16: 8 significant bits
    _, byte = R.quantise(x)
    s = 2.0 ** (byte - 127.0)[:, None]
    hi = R.to_code_value(x / s)
    lo = R.to_code_value((x / s - hi) * 16)
    err = np.abs((hi + lo / 16) * s - x)
    normal = np.abs(x) >= 2.0 ** -6 * s
    assert np.all(err[normal] == 0) and np.all((err <= 2.0 ** -14 * s)[~normal])
    assert _bounds_hold(x, (hi + lo / 16) * s, 0, 2.0 ** -13.8, 2.0 ** -21.8)
    assert not _bounds_hold(x, (hi + lo / 16) * s, 0, 2.0 ** -13.8, 2.0 ** -22)
