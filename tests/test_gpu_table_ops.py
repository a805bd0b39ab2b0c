"""Operators on a vocabulary table against the 64-bit oracle: 4-bit
quantisation, the 4-bit product, token lookup and its gradient.

Tolerances, from the arithmetic:
  quantise   codes, scales and row scales are decided by exact comparisons:
             equal.  The values they stand for have at most 6 significant bits.
  product    terms are exact; products of two terms are exact in fp32 up to the
             block scales' few bits, and at most `d` of them are added in fp32:
             |error| <= d 2^-24 sum |x| |w| in the worst order, taken here as
             16 sqrt(d) 2^-24 of it (adders of an MMA keep 24 bits a step, and the
             order is a tree over 64 columns), plus the output's rounding.
  lookup     one rounding of scale * value in fp32, one to the output type.
  gradient   n fp32 additions: n 2^-24 of the sum of magnitudes, one product, one
             rounding to the output type.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import table_oracle as ora  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
FMT = ("e4m3", "e8m0")
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def sph():
    import __graft_entry__ as g
    g.build()
    from paper_2607_13093_gb300 import sph as mod
    return mod


@pytest.fixture(scope="module")
def ctx(sph):
    c = sph.Context(0)
    yield c
    c.close()


def fmt_id(sph, fmt):
    return sph.SPH_MX4_E4M3 if fmt == "e4m3" else sph.SPH_MX4_E8M0


def f64(t):
    return t.detach().double().cpu().numpy()


def make_x(rows, d, dtype, seed, wide=True):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, d)) * np.exp(rng.standard_normal((rows, 1)))
    if wide:
        x[:, ::37] *= 50
        x[:, 16:32] *= 1e-3
    return torch.tensor(x, dtype=torch.float32).to(dtype).to(DEV)


def held(sph, ctx, V, d, fmt, seed):
    """A table in 4 bits and its decoded values (from the device's bytes)."""
    w = ctx.mx4_quantize(make_x(V, d, torch.float32, seed), fmt_id(sph, fmt))
    return w, decoded(w, fmt)


def decoded(w, fmt):
    nb = -(-w.d // ora.BLOCK[fmt])
    exps = np.zeros(w.codes.shape[0]) if w.row_scale is None else np.log2(f64(w.row_scale))
    return ora.decode(ora.unpack(w.codes.cpu().numpy()), w.scales.cpu().numpy()[:, :nb], exps, w.d,
                      fmt)


def assert_close(got, want, bound, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    off = np.where(np.isnan(want), 0, np.abs(got - want) - bound)
    assert off.max(initial=0) <= 0, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


# ---- quantise -----------------------------------------------------------------
@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 15), (2, 16), (5, 33), (4, 512), (3, 1000),
                                    (2, 1024), (2, 1056), (1, 4097), (2, 8193)])
def test_quantise_equals_the_oracle(sph, ctx, fmt, dtype, rows, d):
    x = make_x(rows, d, dtype, 7 * d + rows, wide=d > 40)
    w = ctx.mx4_quantize(x, fmt_id(sph, fmt))
    back = ctx.mx4_dequantize(w, dtype=torch.float32)
    ctx.sync()
    codes, scales, exps = ora.encode(f64(x), fmt)
    assert np.array_equal(ora.unpack(w.codes.cpu().numpy()), codes)
    got_s = w.scales.cpu().numpy()
    assert np.array_equal(got_s[:, :scales.shape[1]], scales)
    assert (got_s[:, scales.shape[1]:] == 0).all()
    if fmt == "e4m3":
        assert np.array_equal(f64(w.row_scale), 2.0 ** exps)
    else:
        assert w.row_scale is None
    want = ora.decode(codes, scales, exps, d, fmt)
    assert np.array_equal(f64(back), want)
    assert np.array_equal(f64(ctx.mx4_dequantize(w)), want)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [511, 520, 1024, 1040, 2048, 2064, 4096, 4104, 6144, 6160, 8192, 8200,
                               16400])
def test_quantise_row_lengths(sph, ctx, fmt, dtype, d):
    test_quantise_equals_the_oracle(sph, ctx, fmt, dtype, 9, d)


@pytest.mark.parametrize("fmt", FMT)
def test_quantise_midpoints_go_to_the_even_code(sph, ctx, fmt):
    # 6 fixes the scale at one; the rest lie on and beside the midpoints of two codes
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    vals = [6.0] + [v for m in mids for v in (m, np.nextafter(np.float32(m), np.float32(9)),
                                             np.nextafter(np.float32(m), np.float32(0)))]
    for k in (0, -9, 13):
        x = np.zeros((2, 32 * 3), np.float32)
        for i, v in enumerate(vals):
            j = i % 15 + 1 + 16 * (i // 15)
            x[0, j], x[1, j] = v, -v
        x[:, 0::16] = 6.0
        x *= 2.0 ** k
        t = torch.tensor(x, device=DEV)
        w = ctx.mx4_quantize(t, fmt_id(sph, fmt))
        codes, scales, exps = ora.encode(x, fmt)
        assert np.array_equal(ora.unpack(w.codes.cpu().numpy()), codes)


@pytest.mark.parametrize("fmt", FMT)
def test_quantise_extremes(sph, ctx, fmt):
    d = 96
    x = np.random.default_rng(3).standard_normal((8, d)).astype(np.float32)
    x[0] = 0
    x[1] *= 1e-38
    x[2, :] = 1e-42                      # subnormal
    x[3] *= 1e37
    x[4, 40] = np.inf
    x[5, 3], x[5, 90] = np.nan, -np.inf
    x[6, :48] *= 1e-12                   # blocks that underflow beside large ones
    x[7] = np.nan
    t = torch.tensor(x, device=DEV)
    w = ctx.mx4_quantize(t, fmt_id(sph, fmt))
    back = f64(ctx.mx4_dequantize(w, dtype=torch.float32))
    codes, scales, exps = ora.encode(x, fmt)
    assert np.array_equal(w.scales.cpu().numpy()[:, :scales.shape[1]], scales)
    want = ora.decode(codes, scales, exps, d, fmt)
    assert np.array_equal(np.isnan(back), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.array_equal(back[ok], want[ok])


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("off", [0, 1, 3, 8])
def test_quantise_strided_rows_and_given_buffers(sph, ctx, fmt, off):
    wide = make_x(6, 400, torch.bfloat16, 11)
    x = wide[1::2, off:off + 211]
    big = sph.Mx4(torch.full((6, 160), 0xEE, dtype=torch.uint8, device=DEV)[::2],
                  torch.full((6, 32), 0xEE, dtype=torch.uint8, device=DEV)[::2],
                  torch.zeros(3, device=DEV) if fmt == "e4m3" else None, 211, fmt_id(sph, fmt))
    w = ctx.mx4_quantize(x, fmt_id(sph, fmt), out=big)
    ctx.sync()
    codes, scales, _ = ora.encode(f64(x), fmt)
    assert np.array_equal(ora.unpack(w.codes.cpu().numpy())[:, :224], codes)
    assert (w.codes.cpu().numpy()[:, 112:] == 0xEE).all()
    assert np.array_equal(w.scales.cpu().numpy()[:, :scales.shape[1]], scales)
    assert (w.scales.cpu().numpy()[:, 16:] == 0xEE).all()


# ---- product --------------------------------------------------------------------
def product_bound(h, table, fmt, planes, ids, out):
    x, w = np.abs(ora.terms(h, fmt, planes)), np.abs(table if ids is None else table[ids])
    y = ora.product(h, table, fmt, planes, ids)
    return 16 * np.sqrt(h.shape[1]) * 2.0 ** -24 * (x @ w.T) + HALF_ULP[out] * np.abs(y) * 1.01


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("planes", [1, 2, 3, 4])
@pytest.mark.parametrize("rows,V,d", [(1, 128, 64), (1, 1, 1), (3, 130, 33), (16, 300, 256),
                                      (17, 257, 300), (40, 500, 1025)])
def test_product_whole_vocabulary(sph, ctx, fmt, planes, rows, V, d):
    w, table = held(sph, ctx, V, d, fmt, V + d)
    h = make_x(rows, d, torch.float32, rows)
    y = ctx.mx4_logits(h, w, planes=planes)
    ctx.sync()
    want = ora.product(f64(h), table, fmt, planes)
    assert_close(f64(y), want, product_bound(f64(h), table, fmt, planes, None, torch.float32), "y")


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("rows", [2, 31, 129, 260])
@pytest.mark.parametrize("kind", ["runs", "odd", "single", "all"])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_product_of_kept_rows(sph, ctx, fmt, rows, kind, out):
    V, d = 700, 192
    rng = np.random.default_rng(rows)
    ids = {"runs": np.concatenate([np.arange(5, 140), np.arange(200, 264), np.arange(500, 700)]),
           "odd": np.sort(rng.choice(V, 301, replace=False)), "single": np.array([V - 1]),
           "all": np.arange(V)}[kind].astype(np.int32)
    w, table = held(sph, ctx, V, d, fmt, 5)
    wide = make_x(rows, d + 130, torch.bfloat16, 3)
    h = wide[:, 129:129 + d]
    bias = torch.tensor(rng.standard_normal(V), dtype=torch.float32, device=DEV)
    y = ctx.mx4_logits(h, w, keep_ids=torch.tensor(ids, device=DEV), bias=bias, planes=2, dtype=out)
    ctx.sync()
    want = ora.product(f64(h), table, fmt, 2, ids, f64(bias))
    bound = product_bound(f64(h), table, fmt, 2, ids, out) + \
        (HALF_ULP[out] + 2.0 ** -24) * np.abs(f64(bias)[ids]) * 1.01 + 2.0 ** -24 * np.abs(want)
    assert_close(f64(y), want, bound, kind)


@pytest.fixture
def split(request, sph, ctx):
    """The context with CTA pairs and the schedule as asked for."""
    pair, schedule = request.param
    ctx.set_option(sph.SPH_OPT_TC_PAIR, pair)
    ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, schedule)
    yield request.param
    ctx.set_option(sph.SPH_OPT_TC_PAIR, 0)
    ctx.set_option(sph.SPH_OPT_TC_SCHEDULE, 0)


@pytest.mark.parametrize("split", [(1, 1), (1, 2), (2, 1), (2, 2)], indirect=True)
@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("planes", [1, 2, 4])
@pytest.mark.parametrize("rows,V,d,keep", [(1, 100, 300, False), (33, 3000, 1300, True),
                                           (70, 129, 4000, False), (240, 900, 700, True),
                                           (500, 257, 256, False)])
def test_product_on_pairs_and_in_ranges(sph, ctx, split, fmt, planes, rows, V, d, keep):
    rng = np.random.default_rng(rows)
    w, table = held(sph, ctx, V, d, fmt, V + d)
    h = make_x(rows, d, torch.bfloat16, rows)
    ids = None
    if keep:
        ids = np.sort(np.concatenate([np.arange(30, 190), 200 + rng.choice(V - 200, 71,
                                                                           replace=False)]))
        ids = ids.astype(np.int32)
    dev_ids = None if ids is None else torch.tensor(ids, device=DEV)
    y = ctx.mx4_logits(h, w, keep_ids=dev_ids, planes=planes)
    again = ctx.mx4_logits(h, w, keep_ids=dev_ids, planes=planes)
    ctx.sync()
    want = ora.product(f64(h), table, fmt, planes, ids)
    assert_close(f64(y), want, product_bound(f64(h), table, fmt, planes, ids, torch.float32), "y")
    assert torch.equal(y, again)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("planes", [1, 3])
@pytest.mark.parametrize("rows,d,keep", [(1, 10500, True), (32, 10304, False), (40, 10500, True)])
def test_product_of_long_rows(sph, ctx, fmt, planes, rows, d, keep):
    rng = np.random.default_rng(rows)
    w, table = held(sph, ctx, 400, d, fmt, d)
    h = make_x(rows, d, torch.float32, rows)
    ids = np.sort(rng.choice(400, 150, replace=False)).astype(np.int32) if keep else None
    y = ctx.mx4_logits(h, w, keep_ids=None if ids is None else torch.tensor(ids, device=DEV),
                       planes=planes)
    ctx.sync()
    want = ora.product(f64(h), table, fmt, planes, ids)
    assert_close(f64(y), want, product_bound(f64(h), table, fmt, planes, ids, torch.float32), "y")


@pytest.mark.parametrize("fmt", FMT)
def test_product_rows_into_a_wider_buffer(sph, ctx, fmt):
    w, table = held(sph, ctx, 200, 96, fmt, 9)
    h = make_x(5, 96, torch.float16, 2)
    buf = torch.full((5, 333), 7.0, device=DEV)
    y = ctx.mx4_logits(h, w, planes=1, out=buf[:, 3:203])
    ctx.sync()
    want = ora.product(f64(h), table, fmt, 1)
    assert_close(f64(y), want, product_bound(f64(h), table, fmt, 1, None, torch.float32), "y")
    assert (buf[:, :3] == 7).all() and (buf[:, 203:] == 7).all()


@pytest.mark.parametrize("fmt", FMT)
def test_product_nan_stays_in_its_row_and_column(sph, ctx, fmt):
    V, d = 150, 128
    x = make_x(V, d, torch.float32, 4)
    x[17, 40] = float("nan")
    w = ctx.mx4_quantize(x, fmt_id(sph, fmt))
    h = make_x(20, d, torch.float32, 6)
    h[3, 100] = float("inf")
    y = f64(ctx.mx4_logits(h, w, planes=2))
    nan = np.zeros((20, V), bool)
    nan[3], nan[:, 17] = True, True
    assert np.array_equal(np.isnan(y), nan)


def test_more_terms_hold_more_of_the_hidden_states(sph, ctx):
    w, table = held(sph, ctx, 256, 512, "e4m3", 1)
    h = make_x(8, 512, torch.float32, 2, wide=False)
    full = f64(h) @ table.T
    err = [np.linalg.norm(f64(ctx.mx4_logits(h, w, planes=p)) - full) for p in (1, 2, 3, 4)]
    assert all(b < a / 5 for a, b in zip(err, err[1:])), err


def test_product_is_the_same_every_time(sph, ctx):
    w, _ = held(sph, ctx, 3000, 640, "e4m3", 1)
    h = make_x(200, 640, torch.float32, 2)
    first = ctx.mx4_logits(h, w, planes=3).clone()
    for _ in range(3):
        assert torch.equal(ctx.mx4_logits(h, w, planes=3), first)


@pytest.mark.parametrize("pair", [1, 2])
@pytest.mark.parametrize("schedule", [1, 2])
def test_product_waits_give_up(sph, pair, schedule):
    # a wait limit of one cycle runs out somewhere: the call ends, sync reports
    # it, and the context works again with the limit restored
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_TC_PAIR, pair)
    c.set_option(sph.SPH_OPT_TC_SCHEDULE, schedule)
    w, table = held(sph, c, 4000, 4096, "e8m0", 1)
    h = make_x(64, 4096, torch.float32, 2)
    c.mx4_logits(h, w)
    c.sync()
    c.set_option(sph.SPH_OPT_SPIN_LIMIT, 1)
    c.mx4_logits(h, w)
    with pytest.raises(sph.SphError) as e:
        c.sync()
    assert e.value.status == 4
    c.set_option(sph.SPH_OPT_SPIN_LIMIT, 1 << 34)
    y = c.mx4_logits(h, w, planes=1)
    c.sync()
    want = ora.product(f64(h), table, "e8m0", 1)
    assert_close(f64(y), want, product_bound(f64(h), table, "e8m0", 1, None, torch.float32), "y")
    c.close()


# ---- lookup -----------------------------------------------------------------------
@pytest.mark.parametrize("table_type", [torch.float32, torch.bfloat16, torch.float16, *FMT])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (7, 50, 31), (3, 9, 64), (200, 100, 1032),
                                   (2, 5, 2051)])
def test_lookup(sph, ctx, table_type, out, T, V, d):
    rng = np.random.default_rng(T + d)
    tok = rng.integers(0, V, T)
    tok[rng.random(T) < 0.3] = -1
    if table_type in FMT:
        table, values = held(sph, ctx, V, d, table_type, d)
    else:
        table = make_x(V, d, table_type, d)
        values = f64(table)
    scale = float(np.float32(d ** 0.5))
    y = ctx.embed(torch.tensor(tok, dtype=torch.int32, device=DEV), table, scale=scale, dtype=out)
    ctx.sync()
    want = ora.lookup(tok, values, scale)
    # (fp16 results may lie below its normal range, where the grid is 2^-24)
    floor = 2.0 ** -25 if out == torch.float16 else 0
    over = np.abs(want) > 65504 if out == torch.float16 else np.zeros(want.shape, bool)
    got = f64(y)
    assert np.isinf(got[over & (np.abs(want) > 65520)]).all()
    assert_close(np.where(over, 0, got), np.where(over, 0, want),
                 np.abs(want) * (HALF_ULP[out] + 2.0 ** -24) * 1.01 + floor, "lookup")


def test_lookup_of_strided_tables_into_slices(sph, ctx):
    # two halves of a hidden state, each from its own part of a split table
    table = make_x(40, 300, torch.bfloat16, 1)
    tok = torch.tensor([3, 39, 0, 3], dtype=torch.int32, device=DEV)
    out = torch.zeros(4, 300, device=DEV)
    ctx.embed(tok, table[:, :97], out=out[:, :97])
    ctx.embed(tok, table[:, 97:], out=out[:, 97:])
    assert torch.equal(out, table[tok.long()].float())


def test_lookup_and_gradient_report_ids_out_of_range(sph, ctx):
    table = make_x(40, 64, torch.float32, 1)
    tok = torch.tensor([3, 40, 0], dtype=torch.int32, device=DEV)
    y = ctx.embed(tok, table)
    with pytest.raises(sph.SphError) as e:
        ctx.sync()
    assert e.value.status == 1
    assert (y[1] == 0).all() and torch.equal(y[0], table[3])
    g = ctx.embed_grad(tok, torch.ones(3, 64, device=DEV), 40)
    with pytest.raises(sph.SphError) as e:
        ctx.sync()
    assert e.value.status == 1
    assert float(g.sum()) == 2 * 64
    tok[1] = -7
    ctx.embed(tok, table, padding_id=-7)
    ctx.embed_grad(tok, torch.ones(3, 64, device=DEV), 40, padding_id=-7)
    ctx.sync()
    assert tuple(ctx.embed(tok[:0], table).shape) == (0, 64)
    ctx.sync()


@pytest.mark.parametrize("padding", [0, 7, 39])
@pytest.mark.parametrize("T", [6, 3000, 9000])
def test_padding_id_inside_the_vocabulary(sph, ctx, padding, T):
    # its tokens give rows of zeros and take no part in the gradient, whose row stays zero
    rng = np.random.default_rng(T)
    table = make_x(40, 64, torch.float32, 1)
    tok = rng.integers(0, 40, T)
    tok[:3] = padding
    t = torch.tensor(tok, dtype=torch.int32, device=DEV)
    for form, values in ((table, f64(table)), held(sph, ctx, 40, 64, "e4m3", 1)):
        y = ctx.embed(t, form, padding_id=padding, dtype=torch.float32)
        assert np.array_equal(f64(y), ora.lookup(tok, values, 1.0, padding))
    d_out = make_x(T, 64, torch.float32, 2, wide=False)
    for add in (False, True):
        out = torch.full((40, 64), 3.0 if add else float("nan"), device=DEV)
        got = ctx.embed_grad(t, d_out, 40, padding_id=padding, accumulate=add, out=out)
        ctx.sync()
        onto = np.full((40, 64), 3.0) if add else None
        want = ora.gradient(tok, f64(d_out), 40, 1.0, padding, onto)
        assert_close(f64(got), want, grad_bound(tok, f64(d_out), 40, 1.0, torch.float32, onto), "pad")
        assert (got[padding] == (3.0 if add else 0.0)).all()


@pytest.mark.parametrize("off", range(8))
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [5, 8, 23, 250, 1031])
def test_lookup_at_every_alignment(sph, ctx, out, off, d):
    # the other row stride is odd: the rows of a call have every alignment of their own too
    T, V, W = 40, 17, 1047
    tok = np.random.default_rng(off).integers(0, V, T)
    t = torch.tensor(tok, dtype=torch.int32, device=DEV)
    src = torch.full((V, W + 2), float("nan"), dtype=torch.bfloat16, device=DEV)
    src[:, 7 - off:7 - off + d] = make_x(V, d, torch.bfloat16, d)
    for table, values in ((src[:, 7 - off:7 - off + d], f64(src[:, 7 - off:7 - off + d])),
                          held(sph, ctx, V, d, "e4m3", d), held(sph, ctx, V, d, "e8m0", d)):
        buf = torch.full((T, W), 7.0, dtype=out, device=DEV)
        ctx.embed(t, table, out=buf[:, off:off + d])
        ctx.sync()
        assert np.array_equal(f64(buf[:, off:off + d]), ora.lookup(tok, values, 1.0))
        assert (buf[:, :off] == 7).all() and (buf[:, off + d:] == 7).all()


# ---- gradient -----------------------------------------------------------------------
def grad_bound(tok, d_out, V, scale, out, onto=None):
    """Bound of an fp32 sum in any order, and the roundings after it."""
    mag = ora.gradient(tok, np.abs(d_out), V, abs(scale))
    n = np.bincount(np.where((tok < 0) | (tok >= V), V, tok), minlength=V + 1)[:V, None]
    base = 0 if onto is None else np.abs(onto)
    return (n + 2) * 2.0 ** -24 * 1.01 * mag + (HALF_ULP[out] + 2.0 ** -24) * 1.01 * (mag + base)


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (5, 3, 17), (64, 10, 40), (300, 1000, 1032),
                                   (1000, 7, 33)])
def test_gradient(sph, ctx, src, out, add, T, V, d):
    rng = np.random.default_rng(T + V + d)
    tok = np.minimum((V * rng.random(T) ** 3).astype(np.int64), V - 1)
    tok[rng.random(T) < 0.2] = -1
    d_out = make_x(T, d, src, T, wide=False)
    onto = make_x(V, d, out, V, wide=False)
    start = f64(onto)
    got = ctx.embed_grad(torch.tensor(tok, dtype=torch.int32, device=DEV), d_out, V, scale=1.5,
                         accumulate=add, out=onto)
    ctx.sync()
    want = ora.gradient(tok, f64(d_out), V, 1.5, onto=start if add else None)
    floor = 2.0 ** -25 if out == torch.float16 else 0
    assert_close(f64(got), want, floor + grad_bound(tok, f64(d_out), V, 1.5, out,
                                                    start if add else None), "gradient")
    if add:      # rows without a token keep their bits
        none = np.setdiff1d(np.arange(V), tok)
        assert np.array_equal(f64(got)[none], start[none])


@pytest.mark.parametrize("case", ["one id", "two ids", "every id once", "sorted", "all padding",
                                  "boundaries"])
@pytest.mark.parametrize("T", [33, 4097, 20000])
def test_gradient_of_skewed_tokens(sph, ctx, case, T):
    d, V = 24, 70000
    tok = {"one id": np.full(T, 69999), "two ids": np.arange(T) % 2 * 600,
           "every id once": np.random.default_rng(1).permutation(V)[:T],
           "sorted": np.arange(T) // 3, "all padding": np.full(T, -1),
           "boundaries": np.arange(T) // 32 + 511}[case]
    rng = np.random.default_rng(T)
    d_out = torch.tensor(rng.standard_normal((T, d)), dtype=torch.bfloat16, device=DEV)
    t = torch.tensor(tok, dtype=torch.int32, device=DEV)
    got = ctx.embed_grad(t, d_out, V)
    ctx.sync()
    want = ora.gradient(tok, f64(d_out), V, 1.0)
    assert_close(f64(got), want, grad_bound(tok, f64(d_out), V, 1.0, torch.float32), case)
    again = ctx.embed_grad(t, d_out, V)
    assert torch.equal(got, again)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("d,src,out", [(40, torch.bfloat16, torch.float32),
                                       (1032, torch.float32, torch.bfloat16),
                                       (33, torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("add", [False, True])
def test_gradient_of_random_runs(sph, ctx, seed, d, src, out, add):
    # runs of equal ids of every length around the ranges' and the windows' (1 to 140),
    # some ids absent, the tokens shuffled
    rng = np.random.default_rng(seed)
    lengths = rng.choice([1, 2, 7, 8, 9, 15, 16, 17, 18, 31, 32, 33, 34, 64, 65, 140],
                         int(rng.integers(20, 90)))
    ids = np.sort(rng.choice(4000, len(lengths), replace=False))
    tok = rng.permutation(np.concatenate([np.repeat(ids, lengths), np.full(rng.integers(0, 40), -1)]))
    d_out = torch.tensor(rng.standard_normal((len(tok), d)), dtype=src, device=DEV)
    onto = torch.tensor(rng.standard_normal((4000, d)), dtype=out, device=DEV) if add else \
        torch.full((4000, d), float("nan"), dtype=out, device=DEV)
    start = f64(onto)
    got = ctx.embed_grad(torch.tensor(tok, dtype=torch.int32, device=DEV), d_out, 4000, scale=0.75,
                         accumulate=add, out=onto)
    ctx.sync()
    base = start if add else None
    want = ora.gradient(tok, f64(d_out), 4000, 0.75, onto=base)
    assert_close(f64(got), want, grad_bound(tok, f64(d_out), 4000, 0.75, out, base), "runs")


@pytest.mark.parametrize("V,d,T", [(300000, 128, 3000), (99991, 257, 1), (70001, 1024, 9000)])
def test_gradient_fills_every_row_of_a_large_table(sph, ctx, V, d, T):
    # (rows beyond the ones zeroed beside the sort: over 96 MB)
    rng = np.random.default_rng(V)
    tok = rng.integers(0, V, T)
    tok[0] = V - 1
    d_out = torch.tensor(rng.standard_normal((T, d)), dtype=torch.float32, device=DEV)
    out = torch.full((V, d), float("nan"), device=DEV)
    t = torch.tensor(tok, device=DEV)
    ctx.embed_grad(t.int(), d_out, V, out=out)
    ctx.sync()
    want = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, t, d_out.double())
    n = int(np.bincount(tok).max())
    mag = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, t, d_out.double().abs())
    assert bool(((out.double() - want).abs() <= (n + 2) * 2.0 ** -24 * 1.01 * mag).all())


def test_gradient_of_long_lists(sph, ctx):
    # more tokens than the cluster's tiles hold, over ids that need four digits
    T, d, V = 150000, 8, 300_000_007
    rng = np.random.default_rng(0)
    pool = np.sort(rng.choice(V, 500, replace=False))
    pool[-1] = V - 1
    tok = pool[np.minimum((500 * rng.random(T) ** 4).astype(int), 499)]
    d_out = torch.tensor(rng.standard_normal((T, d)), dtype=torch.float32, device=DEV)
    out = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    ctx.embed_grad(torch.tensor(tok, dtype=torch.int32, device=DEV), d_out, V, accumulate=True,
                   out=out)
    ctx.sync()
    rows = torch.tensor(pool, device=DEV)
    small = np.searchsorted(pool, tok)
    want = ora.gradient(small, f64(d_out), 500, 1.0)
    assert_close(f64(out[rows]), want, grad_bound(small, f64(d_out), 500, 1.0, torch.bfloat16),
                 "long")
    assert int((out != 0).any(1).sum()) == len(np.unique(tok))


def test_gradient_of_no_tokens(sph, ctx):
    g = torch.ones(30, 40, device=DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    ctx.embed_grad(none, torch.empty(0, 40, device=DEV), 30, accumulate=True, out=g)
    assert (g == 1).all()
    ctx.embed_grad(none, torch.empty(0, 40, device=DEV), 30, out=g)
    assert (g == 0).all()


def test_gradient_into_unaligned_slices(sph, ctx):
    tok = torch.tensor([4, 1, 4, 0, 29], dtype=torch.int32, device=DEV)
    src = make_x(5, 211, torch.bfloat16, 3)[:, 3:198]
    buf = torch.full((30, 301), 5.0, dtype=torch.bfloat16, device=DEV)
    ctx.embed_grad(tok, src, 30, out=buf[:, 1:196])
    ctx.sync()
    want = ora.gradient(tok.cpu().numpy(), f64(src), 30, 1.0)
    assert_close(f64(buf[:, 1:196]), want,
                 grad_bound(tok.cpu().numpy(), f64(src), 30, 1.0, torch.bfloat16), "slice")
    assert (buf[:, 0] == 5).all() and (buf[:, 196:] == 5).all()


@pytest.mark.parametrize("off", range(8))
@pytest.mark.parametrize("src,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                     (torch.float16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("d", [5, 8, 250, 1031])
def test_gradient_at_every_alignment(sph, ctx, src, out, add, off, d):
    T, V, W = 90, 23, 1047
    tok = np.random.default_rng(off).integers(0, V // 2, T)       # (long and short runs)
    tok[-30:] = V - 1
    t = torch.tensor(tok, dtype=torch.int32, device=DEV)
    rows = torch.full((T, W + 2), float("nan"), dtype=src, device=DEV)
    g = rows[:, 7 - off:7 - off + d]
    g.copy_(make_x(T, d, src, d, wide=False))
    buf = torch.full((V, W), 7.0, dtype=out, device=DEV)
    ctx.embed_grad(t, g, V, accumulate=add, out=buf[:, off:off + d])
    ctx.sync()
    onto = np.full((V, d), 7.0) if add else None
    want = ora.gradient(tok, f64(g), V, 1.0, -1, onto)
    assert_close(f64(buf[:, off:off + d]), want, grad_bound(tok, f64(g), V, 1.0, out, onto), "g")
    assert (buf[:, :off] == 7).all() and (buf[:, off + d:] == 7).all()


def test_gradient_against_differences(sph, ctx):
    # L(W) = sum(C * lookup(W)): dL/dW by central differences in 64 bits of the
    # oracle's lookup, and by the call from dL/dout = C
    rng = np.random.default_rng(5)
    tok = np.array([2, 0, 2, 2, 5])
    W, C = rng.standard_normal((6, 4)), rng.standard_normal((5, 4))
    C32 = torch.tensor(C, dtype=torch.float32, device=DEV)
    got = f64(ctx.embed_grad(torch.tensor(tok, dtype=torch.int32, device=DEV), C32, 6, scale=2.0))
    for v in range(6):
        for c in range(4):
            lo, hi = W.copy(), W.copy()
            lo[v, c] -= 1e-3
            hi[v, c] += 1e-3
            diff = ((f64(C32) * (ora.lookup(tok, hi, 2.0) - ora.lookup(tok, lo, 2.0))).sum()) / 2e-3
            assert abs(got[v, c] - diff) < 1e-5


# ---- offsets past 32 bits, tiny tables ---------------------------------------------
def test_offsets_past_32_bits(sph, ctx):
    V, d = 600_000, 8192                  # 4.9e9 elements; 2.5e9 bytes of codes
    rng = np.random.default_rng(1)
    ids = np.array([0, 5, 262143, 262144, 524288, V - 3, V - 1], np.int32)
    t = torch.tensor(ids, device=DEV)
    rows = make_x(len(ids), d, torch.bfloat16, 3)
    table = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    table[t.long()] = rows
    assert torch.equal(ctx.embed(t, table), rows)
    got = ctx.embed_grad(t, rows, V, out=table, accumulate=True)
    ctx.sync()
    assert torch.equal(got[t.long()], (rows.float() * 2).bfloat16())
    del table, got
    w = sph.mx4_empty(V, d, sph.SPH_MX4_E4M3, DEV)
    few = ctx.mx4_quantize(rows, sph.SPH_MX4_E4M3)
    for dst, src in zip(w[:3], few[:3]):
        dst.zero_()
        dst[t.long()] = src
    values = decoded(few, "e4m3")
    assert np.array_equal(f64(ctx.embed(t, w, dtype=torch.float32)), values)
    h = make_x(3, d, torch.float32, 4)
    for keep in (t, None):
        y = ctx.mx4_logits(h, w, keep_ids=keep, planes=2)
        y = y if keep is not None else y[:, t.long()]
        want = ora.product(f64(h), values, "e4m3", 2)
        assert_close(f64(y), want, product_bound(f64(h), values, "e4m3", 2, None, torch.float32), "y")
    big = torch.zeros(1 << 20, 2304, dtype=torch.bfloat16, device=DEV)       # 2.4e9 elements
    big[-1] = 1
    back = ctx.mx4_dequantize(ctx.mx4_quantize(big))
    ctx.sync()
    ones = ora.decode(*ora.encode(np.ones((1, 2304)), "e4m3"), 2304, "e4m3")
    assert np.array_equal(f64(back[-1:]), ones) and float(back[:-1].abs().max()) == 0


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("V,keep", [(5, [1, 3]), (1, [0]), (33, list(range(33))), (40, [39])])
def test_product_of_tiny_tables(sph, ctx, fmt, V, keep):
    w, table = held(sph, ctx, V, 48, fmt, V)
    h = make_x(2, 48, torch.float32, 1)
    y = ctx.mx4_logits(h, w, keep_ids=torch.tensor(keep, dtype=torch.int32, device=DEV))
    ctx.sync()
    want = ora.product(f64(h), table, fmt, 2, np.array(keep))
    assert_close(f64(y), want,
                 product_bound(f64(h), table, fmt, 2, np.array(keep), torch.float32), "y")


def test_calls_between_the_other_ones(sph, ctx):
    # the context's scratch goes from call to call without a wait between
    w, _ = held(sph, ctx, 3000, 512, "e4m3", 1)
    table = make_x(3000, 512, torch.bfloat16, 2)
    h = make_x(64, 512, torch.float32, 3)
    tok = torch.randint(0, 3000, (5000,), dtype=torch.int32, device=DEV)
    d_out = make_x(5000, 512, torch.bfloat16, 4)
    alone = []
    for call in (lambda: ctx.mx4_logits(h, w), lambda: ctx.embed_grad(tok, d_out, 3000),
                 lambda: ctx.partial_logits(h, table)[0], lambda: ctx.mx4_logits(h[:1], w, planes=4)):
        alone.append((call, call().clone()))
        torch.cuda.synchronize()
    for _ in range(20):
        got = [call() for call, _ in alone]
    torch.cuda.synchronize()
    for g, (_, want) in zip(got, alone):
        assert torch.equal(g, want)


# ---- streams, capture, refusals -------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph(sph, ctx):
    c = sph.Context(0)
    w, table = held(sph, c, 500, 256, "e4m3", 2)
    h = make_x(9, 256, torch.float32, 1)
    tok = torch.tensor([1, 5, 1, 499], dtype=torch.int32, device=DEV)
    y, e, g = (torch.empty(9, 500, device=DEV), torch.empty(4, 256, device=DEV),
               torch.empty(500, 256, device=DEV))
    c.reserve(16, 512, 256)
    torch.cuda.synchronize()

    def calls():
        c.mx4_logits(h, w, out=y)
        c.embed(tok, w, out=e)
        c.embed_grad(tok, e, 500, out=g)

    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, e, g)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for t in (y, e, g):
            t.fill_(-3)
        calls()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, e, g), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for t in (y, e, g):
        t.fill_(-3)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, e, g), want))
    torch.cuda.synchronize()
    c.close()


def test_inputs_written_just_before_the_call(sph, ctx):
    # each call follows the kernel that writes its input, with nothing between
    w, _ = held(sph, ctx, 600, 512, "e8m0", 2)
    h0 = make_x(40, 512, torch.float32, 1)
    want = ctx.mx4_logits(h0 * 2, w).clone()
    torch.cuda.synchronize()
    for _ in range(20):
        h = h0.clone()
        h.mul_(2)
        assert torch.equal(ctx.mx4_logits(h, w), want)


def test_refusals(sph, ctx):
    w, _ = held(sph, ctx, 64, 64, "e4m3", 1)
    h = make_x(4, 64, torch.float32, 1)
    tok = torch.tensor([1], dtype=torch.int32, device=DEV)
    ids = torch.tensor([1, 2], dtype=torch.int32, device=DEV)
    lib = [
        (lambda: ctx.mx4_logits(h, w, planes=0), 1), (lambda: ctx.mx4_logits(h, w, planes=5), 1),
        (lambda: ctx.mx4_logits(h, w, dtype=torch.float16), 2),
        (lambda: ctx.mx4_logits(h, w._replace(row_scale=None)), 1),
        (lambda: ctx.mx4_logits(h, w._replace(format=9)), 1),
        (lambda: ctx.mx4_logits(h[:0], w), 1),
        (lambda: ctx.mx4_logits(h, w._replace(codes=w.codes[:, :31].contiguous()[:, :31])), None),
        (lambda: ctx.embed(tok, h, scale=float("nan")), 1),
        (lambda: ctx.embed_grad(tok, h[:1], 0), 1),
        (lambda: ctx.mx4_logits(h, w, keep_ids=ids[:0]), 1),
    ]
    for call, status in lib:
        with pytest.raises((sph.SphError, ValueError)) as e:
            call()
        if status is not None:
            assert isinstance(e.value, sph.SphError) and e.value.status == status
    host = [
        lambda: ctx.mx4_quantize(h.cpu()), lambda: ctx.mx4_quantize(h.double()),
        lambda: ctx.mx4_quantize(h.t()), lambda: ctx.mx4_quantize(h, 7),
        lambda: ctx.mx4_logits(h[:, :63], w), lambda: ctx.mx4_logits(h, w, keep_ids=ids.long()),
        lambda: ctx.mx4_logits(h, w, bias=torch.zeros(63, device=DEV)),
        lambda: ctx.mx4_logits(h, w, out=torch.empty(4, 63, device=DEV)),
        lambda: ctx.mx4_logits(h, w._replace(scales=w.scales[:, :3])),
        lambda: ctx.embed(tok.long(), h), lambda: ctx.embed(tok.cpu(), h),
        lambda: ctx.embed_grad(tok, h, 64),
        lambda: ctx.embed_grad(tok, h[:1], 64, accumulate=True),
        lambda: ctx.embed_grad(tok, h[:1], 64, out=torch.empty(64, 63, device=DEV)),
    ]
    for call in host:
        with pytest.raises(ValueError):
            call()
    ctx.sync()
