"""What the 8-bit cache's row format promises, from its definition in 64 bits (CPU)."""

import numpy as np

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
