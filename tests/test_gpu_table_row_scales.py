"""The 4-bit product of tables and hidden states whose rows differ by many powers of two: the
row scales of the e4m3 form (2^-110 to 2^116 each) may not take a logit out of fp32's range
that lies within it.

Tolerance as in test_gpu_table_ops.py: 16 sqrt(d) 2^-24 of the sum of magnitudes (which the
scales multiply exactly) and the output's rounding, here with a subnormal result's own step."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import table_oracle as ora  # noqa: E402
from test_gpu_table_ops import HALF_ULP, assert_close, ctx, decoded, f64, product_bound, sph  # noqa: E402,F401

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("pair,schedule", [(2, 1), (2, 2), (1, 1)])
@pytest.mark.parametrize("planes", [1, 2, 4])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_logits_within_range_stay_within(sph, ctx, pair, schedule, planes, out):  # noqa: F811
    V, d, R = 300, 320, 40
    rng = np.random.default_rng(planes)
    w_exp, h_exp = rng.integers(-115, 124, V), rng.integers(-115, 124, R)
    x = rng.standard_normal((V, d)) * 2.0 ** w_exp[:, None]
    w = ctx.mx4_quantize(torch.tensor(x, dtype=torch.float32, device=DEV), sph.SPH_MX4_E4M3)
    table = decoded(w, "e4m3")
    h = torch.tensor(rng.standard_normal((R, d)) * 2.0 ** h_exp[:, None], dtype=torch.float32, device=DEV)
    ctx.set_option(sph.SPH_OPT_TC_PAIR, pair)
    ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, schedule)
    try:
        y = f64(ctx.mx4_logits(h, w, planes=planes, dtype=out))
        ctx.sync()
    finally:
        ctx.set_option(sph.SPH_OPT_TC_PAIR, 0)
        ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, 0)
    want = ora.product(f64(h), table, "e4m3", planes)
    bound = product_bound(f64(h), table, "e4m3", planes, None, out)
    # (bf16 has fp32's exponents, and 7 bits of its subnormal numbers are 2^-133 apart)
    step = 2.0 ** -149 if out == torch.float32 else 2.0 ** -133
    inside, above = np.abs(want) + bound < 2.0 ** 127, np.abs(want) - bound > 2.0 ** 128
    assert 0.4 < inside.mean() and above.mean() > 0.05
    assert_close(np.where(inside, y, 0), np.where(inside, want, 0), bound + step, "logits")
    assert np.array_equal(y[above], np.sign(want[above]) * np.inf)


def test_bias_is_added_to_the_scaled_sum(sph, ctx):  # noqa: F811
    V, d, R = 130, 64, 3
    rng = np.random.default_rng(1)
    w = ctx.mx4_quantize(torch.tensor(rng.standard_normal((V, d)) * 2.0 ** 100, dtype=torch.float32,
                                      device=DEV), sph.SPH_MX4_E4M3)
    h = torch.tensor(rng.standard_normal((R, d)) * 2.0 ** -100, dtype=torch.float32, device=DEV)
    bias = torch.tensor(rng.standard_normal(V), dtype=torch.float32, device=DEV)
    y = f64(ctx.mx4_logits(h, w, bias=bias))
    ctx.sync()
    table = decoded(w, "e4m3")
    want = ora.product(f64(h), table, "e4m3", 2, None, f64(bias))
    bound = product_bound(f64(h), table, "e4m3", 2, None, torch.float32) + \
        HALF_ULP[torch.float32] * 1.01 * (np.abs(f64(bias)) + np.abs(want))
    assert_close(y, want, bound, "bias")


@pytest.mark.parametrize("fmt", ["e4m3", "e8m0"])
@pytest.mark.parametrize("schedule", [1, 2])
@pytest.mark.parametrize("planes", [1, 2, 4])
def test_finite_where_the_magnitudes_add_up_within_range(sph, ctx, fmt, schedule, planes):  # noqa: F811
    # both formats: whatever order the products add in, no part of such a sum leaves the range
    # (terms after the first hold less than a fourth of it); results below the normal range may
    # be off by its start
    V, d, R = 300, 320, 40
    rng = np.random.default_rng(10 + planes)
    w_exp, h_exp = rng.integers(-115, 124, V), rng.integers(-115, 124, R)
    x = rng.standard_normal((V, d)) * 2.0 ** w_exp[:, None]
    w = ctx.mx4_quantize(torch.tensor(x, dtype=torch.float32, device=DEV),
                         sph.SPH_MX4_E4M3 if fmt == "e4m3" else sph.SPH_MX4_E8M0)
    table = decoded(w, fmt)
    h = torch.tensor(rng.standard_normal((R, d)) * 2.0 ** h_exp[:, None], dtype=torch.float32, device=DEV)
    ctx.set_option(sph.SPH_OPT_TC_PAIR, 2)
    ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, schedule)
    try:
        y = f64(ctx.mx4_logits(h, w, planes=planes))
        ctx.sync()
    finally:
        ctx.set_option(sph.SPH_OPT_TC_PAIR, 0)
        ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, 0)
    want = ora.product(f64(h), table, fmt, planes)
    sure = 2 * np.abs(f64(h)) @ np.abs(table).T < 2.0 ** 127
    assert 0.4 < sure.mean() < 0.9
    bound = product_bound(f64(h), table, fmt, planes, None, torch.float32) + 2.0 ** -126
    assert_close(np.where(sure, y, 0), np.where(sure, want, 0), bound, fmt)
