"""Pins of the actor oracle (oracle/actor.py) that do not use the oracle's own arithmetic: rational numbers for the levels,
Python integers for the products, hand-made rows and enumerated shares for the draws."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import actor


def nearest_even(f):
    low = f.numerator // f.denominator
    rest = f - low
    return low + (1 if rest > Fraction(1, 2) or (rest == Fraction(1, 2) and low % 2) else 0)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_levels_are_the_nearest_whole_numbers_to_the_exact_quotients(dtype):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((6, 200)).astype(dtype)
    x[1] = np.round(x[1] * 8) / 16          # many quotients half way between two levels ...
    x[1, 0] = 127.0 / 16
    x[2] = np.round(x[2] * 8) * 1.5         # ... with a largest magnitude that is no power of two
    x[2, 0] = 381.0
    x[3] *= dtype(1e-3)
    x[4] = 0
    x[5, 7] = np.inf
    levels, scales = actor.quantize_rows(x)
    for r in range(4):
        a = max(abs(Fraction(float(v))) for v in x[r])
        assert [nearest_even(127 * Fraction(float(v)) / a) for v in x[r]] == levels[r].tolist()
        assert scales[r] == pytest.approx(float(a / 127), rel=1e-15)
    assert not levels[4].any() and scales[4] == 0 and not levels[5].any() and np.isnan(scales[5])


def test_products_against_python_integers():
    rng = np.random.default_rng(2)
    xq, wq = rng.integers(-128, 128, (3, 50)), rng.integers(-128, 128, (4, 50))
    sx, sw, b = rng.random(3), rng.random(4), rng.standard_normal(4)
    y, z = actor.linear(xq, sx, wq, sw, b), actor.linear(xq, sx, wq, sw, b, relu=True)
    for m in range(3):
        for n in range(4):
            want = sum(int(p) * int(q) for p, q in zip(xq[m], wq[n])) * sx[m] * sw[n] + b[n]
            assert y[m, n] == pytest.approx(want, rel=1e-13, abs=1e-13) and z[m, n] == max(0.0, y[m, n])


def shares(x, steps=4096, **kw):
    """How often each index is drawn over an even grid of u."""
    got = np.zeros(len(x))
    for j in range(steps):
        got[actor.draw(x, (j + 0.5) / steps, **kw).index] += 1
    return got / steps


def test_shares_are_the_filtered_softmax():
    x = np.array([0.3, -1.0, 2.0, 0.3, 1.5])
    soft = lambda keep, t=1.0: np.where(keep, np.exp(x / t), 0) / np.where(keep, np.exp(x / t), 0).sum()  # noqa: E731
    everything = np.ones(5, bool)
    assert np.abs(shares(x) - soft(everything)).max() < 1 / 2048
    assert np.abs(shares(x, temperature=0.5) - soft(everything, 0.5)).max() < 1 / 2048
    assert np.abs(shares(x, top_k=3) - soft(np.array([1, 0, 1, 0, 1], bool))).max() < 1 / 2048      # the tie goes to index 0
    assert np.abs(shares(x, top_k=4) - soft(np.array([1, 0, 1, 1, 1], bool))).max() < 1 / 2048
    p = soft(everything)
    assert np.abs(shares(x, top_p=p[2] * 0.99) - soft(np.array([0, 0, 1, 0, 0], bool))).max() < 1e-9
    assert np.abs(shares(x, top_p=p[2] * 1.01) - soft(np.array([0, 0, 1, 0, 1], bool))).max() < 1 / 2048
    assert np.abs(shares(x, min_p=np.exp(-0.6)) - soft(np.array([0, 0, 1, 0, 1], bool))).max() < 1 / 2048
    # top-p counts within what top-k has left: 0.7 of {2, 4} is 2 and 4, 0.6 of it is 2 alone
    assert actor.draw(x, 0.999, top_k=2, top_p=0.7).index == 4 and actor.draw(x, 0.999, top_k=2, top_p=0.6).index == 2


def test_draws_where_nothing_is_left_and_at_the_ends():
    inf, nan = np.inf, np.nan
    for bad in (dict(temperature=-1.0), dict(temperature=nan), dict(temperature=inf), dict(top_p=nan), dict(min_p=nan)):
        assert actor.draw([1.0, 2.0], 0.5, **bad).index == -1
    assert actor.draw([1.0, nan], 0.5).index == -1 and actor.draw([-inf, -inf], 0.5).index == -1 and actor.draw([], 0.5).index == -1
    assert actor.draw([1.0, 2.0], nan).index == -1
    assert actor.draw([3.0, 5.0, 5.0], 0.9, temperature=0.0)[:2] == (1, 0.0)
    assert actor.draw([-inf, 0.0, 0.0], 0.0).index == 1 and actor.draw([0.0, 0.0, -inf], 5.0).index == 1
    assert actor.draw([inf, 7.0, inf], 0.5).index == 2 and actor.draw([inf, 7.0, inf], 0.25).logp == pytest.approx(np.log(0.5))
    assert actor.draw([0.0] * 4, 0.5).index == 2 and actor.draw([0.0] * 4, np.nextafter(0.5, 0)).index == 1
    assert actor.draw([0.0] * 4, 0.99, top_p=0.5).index == 1 and actor.draw([0.0] * 4, 0.99, top_p=0.0).index == 0
    assert actor.draw([0.0] * 4, 0.99, top_k=3).index == 2
