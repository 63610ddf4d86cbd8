"""The 4-bit cache's oracle against rational arithmetic and closed forms."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv4


def _code_rational(x, lo, s):
    if s == 0:
        return 0
    q = (Fraction(x) - Fraction(lo)) / Fraction(s) + Fraction(1, 2)
    return min(15, q.numerator // q.denominator)


@pytest.mark.parametrize("scale", [1e-6, 0.01, 1.0, 37.0, 60000.0])
def test_codes_by_rational_arithmetic(scale):
    rng = np.random.default_rng(5)
    x = np.clip(rng.standard_normal((20, 64)) * scale, -60000, 60000)
    x = (np.round(x / scale * 64) / 64 * scale).astype(np.float16).astype(np.float64)
    c, s, lo = kv4.quantise(x)
    for i in range(20):
        for g in range(2):
            v = x[i, 32 * g:32 * g + 32]
            assert lo[i, g] == v.min()
            span = Fraction(v.max()) - Fraction(v.min())
            step = Fraction(float(np.spacing(np.float16(s[i, g]))))
            assert abs(Fraction(s[i, g]) - span / 15) <= step / 2
            for j in range(32):
                assert c[i, 32 * g + j] == _code_rational(v[j], lo[i, g], s[i, g])


def test_ties_round_up_and_extremes_keep_their_place():
    x = np.zeros(32)
    x[:6] = [0.0, 15.0, 0.5, 1.5, 6.5, 7.49]                 # s = 1
    c, s, lo = kv4.quantise(x)
    assert s[0] == 1.0 and lo[0] == 0.0
    assert list(c[:6]) == [0, 15, 1, 2, 7, 7]
    assert np.array_equal(kv4.held(x)[:2], [0.0, 15.0])


def test_constant_and_bad_groups():
    assert np.array_equal(kv4.held(np.full(32, -3.5)), np.full(32, -3.5))
    for bad in (np.nan, np.inf, -np.inf, 65536.0):
        x = np.zeros(64)
        x[40] = bad
        h = kv4.held(x)
        assert np.array_equal(h[:32], np.zeros(32)) and np.isnan(h[32:]).all()


def test_error_of_the_format():
    """Within s / 2 plus the rounding of 15 s, s itself off by 2^-11 at most."""
    x = np.random.default_rng(1).standard_normal((50, 128)).astype(np.float16).astype(np.float64)
    _, s, _ = kv4.quantise(x)
    bound = np.repeat(s * (0.5 + 15 * 2.0 ** -11), 32, axis=-1)
    assert (np.abs(kv4.held(x) - x) <= bound).all()


def test_attend_against_loops():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((4, 32)), rng.standard_normal((2, 9, 32)), rng.standard_normal((2, 9, 32))
    seen = np.array([1, 1, 0, 1, 1, 1, 0, 1, 1], bool)
    add = rng.standard_normal(9)
    out, tol = kv4.attend(q, k, v, seen, add)
    for h in range(4):
        num, den = np.zeros(32), 0.0
        for j in range(9):
            if seen[j]:
                w = np.exp(sum(q[h, i] * k[h // 2, j, i] for i in range(32)) / 32 ** 0.5 + add[j])
                num, den = num + w * v[h // 2, j], den + w
        assert np.allclose(out[h], num / den, rtol=1e-12, atol=0)
    assert (tol > 0).all() and (tol < 0.02).all()
    out, _ = kv4.attend(q, k, v, np.zeros(9, bool))
    assert not out.any()
