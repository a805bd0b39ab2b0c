"""The 4-bit product where every CTA takes several tiles one after another (its accumulators,
stages and scale sets go round between them), and how far it is from 64 bits.

Tolerances:
  tiles     as in test_gpu_table_ops.py: 16 sqrt(d) 2^-24 of the sum of magnitudes, and the
            output's rounding.
  accuracy  in norm over all logits, 4 x 2^-24: the first two terms' products mostly fit the 24
            bits that an accumulator keeps, so what is left is the roundings of either
            accumulator's last addition, of their sum, and of the scaled result, half a unit
            of 2^-23 each at most.  (Four terms in one accumulator are some 50 x 2^-24 off.)"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import table_oracle as ora  # noqa: E402
from test_gpu_table_ops import HALF_ULP, ctx, decoded, f64, fmt_id, make_x, sph  # noqa: E402,F401

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def up(a):
    return torch.tensor(a, dtype=torch.float64, device=DEV)


@pytest.fixture
def paired(request, sph, ctx):  # noqa: F811
    """Whole tiles, on CTA pairs (1) or single CTAs (2)."""
    ctx.set_option(sph.SPH_OPT_TC_PAIR, request.param)
    ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, 1)
    yield request.param
    ctx.set_option(sph.SPH_OPT_TC_PAIR, 0)
    ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, 0)


# ---- several tiles a CTA --------------------------------------------------------
V, D = 100_000, 320          # 782 tiles of 128 rows: five a CTA; kept ids 586, four


@pytest.fixture(scope="module", params=["e4m3", "e8m0"])
def large(request, sph, ctx):  # noqa: F811
    fmt = request.param
    w = ctx.mx4_quantize(make_x(V, D, torch.float32, 1), fmt_id(sph, fmt))
    rng = np.random.default_rng(2)
    scattered = np.sort(rng.choice(V // 2, V // 4, replace=False))        # then all of the rest
    ids = np.concatenate([scattered, np.arange(V // 2, V)]).astype(np.int32)
    return fmt, w, up(decoded(w, fmt)), torch.tensor(ids, device=DEV)


@pytest.mark.parametrize("paired", [1, 2], indirect=True)
@pytest.mark.parametrize("planes", [1, 2, 3, 4])
@pytest.mark.parametrize("rows", [8, 150, 400])
@pytest.mark.parametrize("keep", [False, True])
def test_many_tiles_a_cta(ctx, large, paired, planes, rows, keep):  # noqa: F811
    fmt, w, table, ids = large
    h = make_x(rows, D, torch.float32, rows)
    bias = torch.randn(V, device=DEV)
    y = ctx.mx4_logits(h, w, keep_ids=ids if keep else None, bias=bias, planes=planes)
    ctx.sync()
    x = up(ora.terms(f64(h), fmt, planes))
    b = bias.double()
    if keep:
        table, b = table[ids.long()], b[ids.long()]
    want = x @ table.T
    bound = 16 * D ** 0.5 * 2.0 ** -24 * (x.abs() @ table.abs().T) + \
        HALF_ULP[torch.float32] * 1.01 * (2 * want.abs() + b.abs())
    off = (y.double() - (want + b)).abs() - bound
    assert bool((off <= 0).all()), (float(off.max()), int((off > 0).sum()))


# ---- accuracy ---------------------------------------------------------------------
@pytest.mark.parametrize("paired", [1, 2], indirect=True)
@pytest.mark.parametrize("fmt", ["e4m3", "e8m0"])
@pytest.mark.parametrize("planes", [1, 2, 3, 4])
@pytest.mark.parametrize("rows,d", [(16, 4608), (300, 4608), (64, 1000)])
def test_error_against_64_bits(sph, ctx, paired, fmt, planes, rows, d):  # noqa: F811
    g = torch.Generator(device=DEV).manual_seed(d + rows)
    w = ctx.mx4_quantize(torch.randn(1500, d, generator=g, device=DEV) * 0.02, fmt_id(sph, fmt))
    h = torch.randn(rows, d, generator=g, device=DEV)
    y = ctx.mx4_logits(h, w, planes=planes)
    ctx.sync()
    want = up(ora.terms(f64(h), fmt, planes)) @ up(decoded(w, fmt)).T
    err = float((y.double() - want).norm() / want.norm())
    assert err <= 4 * 2.0 ** -24, err
