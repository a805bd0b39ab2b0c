"""Pins of the 64-bit oracle of the table operators (no GPU needed): the formats'
tables, nearest codes by exhaustive search, what a term leaves, and the product,
lookup and gradient against plain loops."""
import numpy as np
import pytest

from oracle import table_oracle as ora


def test_e2m1_and_e4m3_tables():
    # e2m1: 1 bit of mantissa, exponent bias 1; e4m3: 3 bits, bias 7, 448 the largest
    e2m1 = [m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1) for e in range(4) for m in range(2)]
    assert list(ora.E2M1) == e2m1
    t = ora.e4m3_table()
    assert t[0] == 0 and t[1] == 2.0 ** -9 and t[8] == 2.0 ** -6 and t[56] == 1 and t[-1] == 448
    assert (np.diff(t) > 0).all()


def test_nearest_takes_the_even_of_two_as_near():
    mids = (ora.E2M1[1:] + ora.E2M1[:-1]) / 2
    got = ora.nearest(mids, ora.E2M1)
    assert (got % 2 == 0).all()
    rng = np.random.default_rng(0)
    v = rng.uniform(0, 8, 2000)
    best = np.abs(v[:, None] - ora.E2M1).min(1)
    assert np.allclose(np.abs(v - ora.E2M1[ora.nearest(v, ora.E2M1)]), best, rtol=0, atol=0)


def test_row_exponent_is_the_least_that_holds_the_row():
    for a in [1e-20, 0.3, 2688.0, np.nextafter(2688.0, 3000), 5376.0, 1e30]:
        k = int(ora.row_exponent(np.array([a]))[0])
        assert a <= 2688 * 2.0 ** k and a > 2688 * 2.0 ** (k - 1)
    assert ora.row_exponent(np.array([0.0]))[0] == 0
    assert list(ora.row_exponent(np.array([1e-44, 3e38]))) == [-110, 116]


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_codes_by_exhaustive_search(fmt):
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((3, 70)) * np.exp(3 * rng.standard_normal((3, 70)))).astype(np.float32)
    codes, scales, exps = ora.encode(x, fmt)
    values = ora.decode(codes, scales, exps, 70, fmt)
    for r in range(3):
        for i in range(scales.shape[1]):
            lo, hi = i * ora.BLOCK[fmt], min(70, (i + 1) * ora.BLOCK[fmt])
            amax = np.abs(x[r, lo:hi]).astype(np.float64).max()
            step = ora._E4M3[scales[r, i]] * 2.0 ** exps[r] if fmt == "e4m3" \
                else 2.0 ** (int(scales[r, i]) - 127)
            if fmt == "e8m0":
                assert step == 2.0 ** max(-126, np.floor(np.log2(amax)) - 2)
            for c in range(lo, hi):
                best = min(abs(abs(float(x[r, c])) - step * q) for q in ora.E2M1)
                assert abs(values[r, c] - float(x[r, c])) == best
    assert (codes[:, 70:] == 0).all()


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_values_have_six_significant_bits(fmt):
    x = np.random.default_rng(2).standard_normal((4, 64))
    c, s, e = ora.encode(x, fmt)
    v = ora.decode(c, s, e, 64, fmt)
    m, _ = np.frexp(v)
    assert (m * 64 == np.round(m * 64)).all()


def test_terms_leave_less_and_less():
    x = np.random.default_rng(3).standard_normal((5, 100))
    left = [np.linalg.norm(x - ora.terms(x, "e4m3", p)) for p in (1, 2, 3, 4)]
    assert all(b < a / 4 for a, b in zip(left, left[1:]))


def test_a_block_with_a_nan_stands_for_nan():
    x = np.ones((1, 64))
    x[0, 20] = np.inf
    for fmt, lo, hi in (("e4m3", 16, 32), ("e8m0", 0, 32)):
        v = ora.decode(*ora.encode(x, fmt)[:2], ora.encode(x, fmt)[2], 64, fmt)
        assert np.isnan(v[0, lo:hi]).all() and np.isfinite(np.delete(v[0], range(lo, hi))).all()


def test_product_lookup_and_gradient_by_loops():
    rng = np.random.default_rng(4)
    h, table = rng.standard_normal((2, 40)), rng.standard_normal((9, 40))
    ids, bias = np.array([1, 4, 8]), rng.standard_normal(9)
    y = ora.product(h, table, "e4m3", 2, ids, bias)
    t = ora.terms(h, "e4m3", 2)
    for r in range(2):
        for j, v in enumerate(ids):
            assert abs(y[r, j] - (sum(t[r, c] * table[v, c] for c in range(40)) + bias[v])) < 1e-12
    tok = [3, -1, 3, 8, 11]
    out = ora.lookup(tok, table, 0.5)
    assert (out[1] == 0).all() and (out[4] == 0).all() and np.array_equal(out[0], 0.5 * table[3])
    d = rng.standard_normal((5, 40))
    g = ora.gradient(tok, d, 9, 0.5)
    assert np.allclose(g[3], 0.5 * (d[0] + d[2]), rtol=0, atol=1e-15)
    assert np.array_equal(g[8], 0.5 * d[3]) and (np.delete(g, [3, 8], axis=0) == 0).all()
