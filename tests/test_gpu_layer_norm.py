"""Layer norm and its gradients against the 64-bit oracle.

Tolerances, from the arithmetic (u = 2^-24, K = 64 additions at most on a value's way into a
sum of a row: up to 32 in a thread, or d / 8192 pieces of 8, then two trees of a block):
  mean   K u mean|x|
  y      n = (x - mean) rstd; the variance is within (K + 6) u of that about the mean used,
         which adds the square of the mean's error; 4 roundings, then weight and bias
  dx     sums K u each of their terms' magnitudes, 8 roundings
  dw     at most rows + 64 additions of products that carry 4 roundings
and the results' own roundings (half a step of the type).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import rows_oracle as ora  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, K = 2.0 ** -24, 64
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


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


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def rows_of(R, d, dtype, seed, wide=0, offset=0.3):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, d + wide)) * np.exp(rng.standard_normal((R, 1))) + offset
    x[:, ::37] *= 20
    return torch.tensor(x, dtype=torch.float32).to(dtype).to(DEV)[:, wide:]


def params(d, dtype, seed):
    rng = np.random.default_rng(seed)
    t = lambda v: torch.tensor(v, dtype=torch.float32).to(dtype).to(DEV)
    return t(1 + 0.3 * rng.standard_normal(d)), t(rng.standard_normal(d))


def check_y(y, x, w, b, centre, eps, out):
    want, mean, rstd = ora.norm(f64(x), f64(w), f64(b), eps, centre)
    X = f64(x)
    w64 = 1.0 if w is None else np.abs(f64(w))
    b64 = 0.0 if b is None else np.abs(f64(b))
    r, off = rstd[:, None], np.abs(X - mean[:, None])
    dm = K * U * np.abs(X).mean(1, keepdims=True) if centre else 0.0
    bound = w64 * r * (dm + off * ((0.5 * (K + 6) + 4) * U + (dm * r) ** 2)) * 1.01
    bound = bound + 3 * U * (w64 * off * r + b64) + HALF[out] * np.abs(want) * 1.01 + LEAST[out]
    assert (np.abs(f64(y) - want) <= bound).all()
    return mean, rstd


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 256), (9, 257), (4, 512), (700, 512), (3, 1000), (650, 1000),
          (2, 1024), (1, 4096), (400, 4096), (5, 4001), (330, 4001), (2, 8192), (310, 8192), (2, 8200),
          (1, 16384), (2, 16389), (1, 40000)]


@pytest.mark.parametrize("R,d", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_any_length(ctx, R, d, dtype):
    x = rows_of(R, d, dtype, R + d)
    w, b = params(d, torch.float32, d)
    y, mean, rstd = ctx.layer_norm(x, w, b, stats=True)
    ctx.sync()
    m64, r64 = check_y(y, x, w, b, True, 1e-5, dtype)
    assert y.dtype == dtype
    X = np.abs(f64(x))
    dm = K * U * X.mean(1)
    assert (np.abs(f64(mean) - m64) <= dm + U * np.abs(m64)).all()
    rel = (0.5 * (K + 6) + 4) * U + (dm * r64) ** 2
    assert (np.abs(f64(rstd) - r64) <= 1.01 * rel * r64).all()


@pytest.mark.parametrize("d", [33, 600, 4096, 9000])
@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("which", ["both", "weight", "bias", "none"])
def test_parameters_and_types(ctx, d, centre, out, which):
    x = rows_of(6, d, torch.bfloat16, d)
    for pt in TYPES:
        w, b = params(d, pt, d)
        w = w if which in ("both", "weight") else None
        b = b if which in ("both", "bias") else None
        y, mean, rstd = ctx.layer_norm(x, w, b, centre=centre, eps=1e-3, stats=True, dtype=out)
        ctx.sync()
        assert (mean is None) == (not centre)
        check_y(y, x, w, b, centre, 1e-3, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [40, 700, 4097])
@pytest.mark.parametrize("wide", [0, 1, 3, 8])
def test_strides_and_alignments(ctx, dtype, d, wide):
    x = rows_of(9, d, dtype, d, wide=wide)
    w, b = params(d + 1, torch.float32, 3)
    for off in (0, 1):
        out = torch.full((9, d + 5), 7.0, dtype=torch.bfloat16, device=DEV)
        y = ctx.layer_norm(x[::2], w[off:off + d], b[off:off + d], out=out[::2, 2:d + 2])
        ctx.sync()
        check_y(y, x[::2], w[off:off + d], b[off:off + d], True, 1e-5, torch.bfloat16)
        assert (out[:, :2] == 7).all() and (out[:, d + 2:] == 7).all() and (out[1::2] == 7).all()


def test_in_place_and_equal_rows(ctx):
    for d in (64, 1000, 4096, 4097, 20000):
        x = rows_of(7, d, torch.bfloat16, d)
        x[3] = 2.5                                # no variance: the bias alone
        w, b = params(d, torch.float32, d)
        want = ctx.layer_norm(x, w, b)
        same = x.clone()
        assert ctx.layer_norm(same, w, b, out=same) is same
        ctx.sync()
        assert torch.equal(same, want) and torch.equal(want[3], b.to(torch.bfloat16))


def test_large_means_leave_the_variance(ctx):
    # a mean 1000 times the spread: E[x^2] - mean^2 would lose ten bits
    rng = np.random.default_rng(0)
    x = torch.tensor(1000 + rng.standard_normal((4, 4096)), dtype=torch.float32, device=DEV)
    y = ctx.layer_norm(x)
    check_y(y, x, None, None, True, 1e-5, torch.float32)
    assert abs(float(y.double().std()) - 1) < 1e-3


def test_nan_and_infinity_stay_in_their_rows(ctx):
    for d in (64, 2000, 5000, 20000):
        x = rows_of(4, d, torch.float32, d)
        want = ctx.layer_norm(x)
        x[1, d // 2], x[2, 0] = float("nan"), float("inf")
        y = ctx.layer_norm(x)
        dy = torch.ones_like(x)
        _, mean, rstd = ctx.layer_norm(x, stats=True)
        dx, _, db = ctx.layer_norm_grad(dy, x, None, mean, rstd)
        ctx.sync()
        assert torch.equal(y[[0, 3]], want[[0, 3]]) and y[1].isnan().all() and y[2].isnan().any()
        assert torch.isfinite(dx[[0, 3]]).all() and dx[1].isnan().all() and (db == 4).all()


# ---- gradients -----------------------------------------------------------------
def check_grads(got, dy, x, w, mean, rstd, types, onto=(0.0, 0.0)):
    dx, dw, db = got
    R, d = x.shape
    Y, X, r = f64(dy), f64(x), f64(rstd)[:, None]
    want = ora.norm_grads(Y, X, f64(w), f64(mean), f64(rstd))
    n = (X if mean is None else X - f64(mean)[:, None]) * r
    g = np.abs(Y if w is None else Y * f64(w))
    gn = np.abs(g * n).mean(1, keepdims=True)
    g1 = g.mean(1, keepdims=True) if mean is not None else 0.0
    bound = r * ((K + 8) * U * (g1 + np.abs(n) * gn) + 8 * U * (g + g1 + np.abs(n) * gn))
    assert (np.abs(f64(dx) - want[0]) <=
            bound + HALF[types[0]] * np.abs(want[0]) * 1.01 + LEAST[types[0]]).all()
    for t, mag, exact, base in ((dw, np.abs(Y * n).sum(0), want[1], onto[0]),
                                (db, np.abs(Y).sum(0), want[2], onto[1])):
        if t is not None:
            off = np.abs(f64(t) - (exact + base))
            assert (off <= (R + K + 6) * U * mag + U * np.abs(exact + base) +
                    HALF[types[1]] * np.abs(exact + base) * 1.01 + LEAST[types[1]]).all()


@pytest.mark.parametrize("R,d", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_rows_of_any_length(ctx, R, d, dtype):
    x, dy = rows_of(R, d, dtype, R + d), rows_of(R, d, dtype, R + d + 1, offset=0.1)
    w, b = params(d, torch.float32, d)
    _, mean, rstd = ctx.layer_norm(x, w, b, stats=True)
    got = ctx.layer_norm_grad(dy, x, w, mean, rstd)
    ctx.sync()
    check_grads(got, dy, x, w, mean, rstd, (dtype, torch.float32))
    again = ctx.layer_norm_grad(dy, x, w, mean, rstd)
    ctx.sync()
    assert all(torch.equal(a.view(torch.uint8), c.view(torch.uint8)) for a, c in zip(got, again))


@pytest.mark.parametrize("R,d", [(5000, 40), (5000, 256), (2600, 512), (2000, 1000), (900, 1536),
                                 (950, 4096), (701, 4104), (330, 5120), (320, 8192), (310, 12000)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", ["both", "none"])
def test_many_rows_and_parameters_of_their_type(ctx, R, d, dtype, which):
    # more rows than blocks, so that each takes several; all of one type
    def equal(one, two):
        return all((a is None and c is None) or torch.equal(a.view(torch.uint8), c.view(torch.uint8))
                   for a, c in zip(one, two))

    def grads(dy, x, d_x=None):
        sums = dict(d_bias=torch.empty(d, device=DEV))
        if w is not None:
            sums["d_weight"] = torch.empty(d, device=DEV)
        return ctx.layer_norm_grad(dy, x, w, mean, rstd, d_x=d_x, **sums)

    x, dy = rows_of(R, d, dtype, R + d), rows_of(R, d, dtype, R + d + 1, offset=0.1)
    w, b = params(d, dtype, d) if which == "both" else (None, None)
    y, mean, rstd = ctx.layer_norm(x, w, b, stats=True)
    got, again = grads(dy, x), grads(dy, x)
    ctx.sync()
    check_y(y, x, w, b, True, 1e-5, dtype)
    check_grads(got, dy, x, w, mean, rstd, (dtype, torch.float32))
    assert equal(got, again)
    # in place of the rows, and of their gradient
    at_x, at_dy = x.clone(), dy.clone()
    assert equal(got, grads(dy, at_x, at_x)) and equal(got, grads(at_dy, x, at_dy))
    ctx.layer_norm(x, w, b, out=x)
    ctx.sync()
    assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_in_place_needs_the_same_form(sph, ctx):
    x = rows_of(4, 64, torch.float32, 1)
    _, mean, rstd = ctx.layer_norm(x, stats=True)
    was, half = x.clone(), x.view(torch.bfloat16)[:, :64]
    wide = x.view(-1)[:3 * 64].view(3, 64)
    for call in (lambda: ctx.layer_norm(x, out=half), lambda: ctx.layer_norm(wide[:2], out=x[::2]),
                 lambda: ctx.layer_norm_grad(x, was, None, mean, rstd, d_x=half),
                 lambda: ctx.layer_norm_grad(was, x, None, mean, rstd, d_x=half)):
        with pytest.raises(sph.SphError):
            call()
    ctx.sync()
    assert torch.equal(x, was)
    ctx.layer_norm(x[:1], out=x[::4])                # one row: any stride
    ctx.sync()


@pytest.mark.parametrize("d", [33, 600, 4096, 9000])
@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("xt,yt,ot,gt", [(0, 1, 2, 0), (1, 0, 1, 1), (2, 1, 0, 2), (1, 2, 1, 0)])
def test_gradients_of_mixed_types(ctx, d, centre, xt, yt, ot, gt):
    x, dy = rows_of(11, d, TYPES[xt], d), rows_of(11, d, TYPES[yt], d + 1)
    for wt in TYPES:
        w, _ = params(d, wt, d)
        _, mean, rstd = ctx.layer_norm(x, w, centre=centre, stats=True)
        got = ctx.layer_norm_grad(dy, x, w, mean, rstd, dtype=TYPES[ot], grad_dtype=TYPES[gt])
        ctx.sync()
        assert got[0].dtype == TYPES[ot] and got[1].dtype == got[2].dtype == TYPES[gt]
        check_grads(got, dy, x, w, mean, rstd, (TYPES[ot], TYPES[gt]))


@pytest.mark.parametrize("d", [40, 700, 4097, 9001])
def test_gradients_of_strided_rows_in_place_and_added(ctx, d):
    for wide in (1, 8):
        x, dy = rows_of(13, d, torch.bfloat16, d, wide), rows_of(13, d, torch.bfloat16, 5, wide)
        w, _ = params(d, torch.float32, d)
        _, mean, rstd = ctx.layer_norm(x, w, stats=True)
        want = ctx.layer_norm_grad(dy, x, w, mean, rstd)
        check_grads(want, dy, x, w, mean, rstd, (torch.bfloat16, torch.float32))
        # onto what the gradients hold
        dw, db = torch.ones(d, device=DEV), torch.full((d,), -2.0, device=DEV)
        got = ctx.layer_norm_grad(dy, x, w, mean, rstd, accumulate=True, d_weight=dw, d_bias=db)
        ctx.sync()
        assert got[1] is dw and got[2] is db
        check_grads(got, dy, x, w, mean, rstd, (torch.bfloat16, torch.float32), (1.0, -2.0))
        # dx where dy or x was
        for k in (0, 1):
            a = [dy.clone(), x.clone()]
            got = ctx.layer_norm_grad(a[0], a[1], w, mean, rstd, d_x=a[k])
            ctx.sync()
            assert got[0] is a[k]
            for p, q in zip(got, want):
                assert torch.equal(p, q)


def test_what_is_left_out_and_no_rows(ctx):
    d = 500
    x, dy = rows_of(20, d, torch.float32, 1), rows_of(20, d, torch.float32, 2)
    w, _ = params(d, torch.float32, 3)
    _, mean, rstd = ctx.layer_norm(x, w, stats=True)
    full = ctx.layer_norm_grad(dy, x, w, mean, rstd)
    for weight, bias in ((w, False), (None, True), (None, False)):
        got = ctx.layer_norm_grad(dy, x, weight, mean, rstd, bias=bias)
        ctx.sync()
        assert (got[1] is None) == (weight is None) and (got[2] is None) == (not bias)
        if weight is not None:
            assert torch.equal(got[0], full[0]) and torch.equal(got[1], full[1])
        if bias:
            assert torch.equal(got[2], full[2])
    for dd in (4, 600, 9000):
        e = torch.empty(0, dd, device=DEV)
        y, m, r = ctx.layer_norm(e, stats=True)
        assert tuple(y.shape) == (0, dd) and m.numel() == r.numel() == 0
        dx, dw, db = ctx.layer_norm_grad(e, e, torch.ones(dd, device=DEV), m, r)
        ctx.sync()
        assert dx.numel() == 0 and (dw == 0).all() and (db == 0).all()
        dw.fill_(3.0)
        ctx.layer_norm_grad(e, e, torch.ones(dd, device=DEV), m, r, accumulate=True, d_weight=dw,
                            d_bias=db)
        ctx.sync()
        assert (dw == 3).all()


def test_gradients_against_differences(ctx):
    # the kernels' own forward pass, in directions: fp32 values of order 1, step 2^-7
    d, R = 300, 5
    x, dy = rows_of(R, d, torch.float32, 1), rows_of(R, d, torch.float32, 2)
    w, b = params(d, torch.float32, 3)
    _, mean, rstd = ctx.layer_norm(x, w, b, stats=True)
    grads = ctx.layer_norm_grad(dy, x, w, mean, rstd)
    for k in range(3):
        g = torch.Generator(device=DEV).manual_seed(k)
        args = [x, w, b]
        way = torch.randn(args[k].shape, generator=g, device=DEV)
        h = 2.0 ** -7 * float(x.std() if k == 0 else 1.0)
        vals = []
        for s in (h, -h):
            moved = list(args)
            moved[k] = args[k] + s * way
            vals.append((ctx.layer_norm(*moved).double() * dy.double()).sum())
        slope = float((vals[0] - vals[1]) / (2 * h))
        want = float((grads[k].double() * way.double()).sum())
        scale = float((grads[k].double() * way.double()).abs().sum())
        # the third derivative's share is h^2 / 6 of the terms' size, rounding u / h
        assert abs(slope - want) <= (2.0 ** -14 + 2.0 ** -16) * 40 * scale


def test_far_rows(ctx):
    # offsets past 2^31 elements, one row at each end
    R, d = (1 << 20) + 5, 2100
    x = torch.empty(R, d, dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    w, b = params(d, torch.float32, 3)
    y, mean, rstd = ctx.layer_norm(x, w, b, stats=True)
    ctx.sync()
    ends = torch.tensor([0, 1, R - 2, R - 1], device=DEV)
    check_y(y[ends], x[ends], w, b, True, 1e-5, torch.bfloat16)
    dx, dw, db = ctx.layer_norm_grad(y, x, w, mean, rstd)
    ctx.sync()
    r64 = rstd[ends].double()
    n = (x[ends].double() - mean[ends].double()[:, None]) * r64[:, None]
    g = y[ends].double() * w.double()
    want = r64[:, None] * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    assert ((dx[ends].double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 1e-4).all()
    # sums of 2^20 rows: blocks add some 2^10 each, then 2^8 to 2^10 blocks
    total = torch.zeros(d, dtype=torch.float64, device=DEV)
    mag = torch.zeros(d, dtype=torch.float64, device=DEV)
    for a in range(0, R, 1 << 17):
        total += y[a:a + (1 << 17)].double().sum(0)
        mag += y[a:a + (1 << 17)].double().abs().sum(0)
    assert ((db.double() - total).abs() <= 4096 * U * mag).all()


@pytest.mark.parametrize("d", [2100, 2104])
def test_the_weights_gradient_over_far_rows(ctx, d):
    # 2^20 rows and offsets past 2^31 elements, rows off 16 bytes and on them: blocks add some
    # 2^11 rows each (152 SMs, three or four blocks an SM), then come 2^9 blocks; in each term
    # one rounding for the difference and one for the product
    R = (1 << 20) + 5
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.empty(R, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    dy = torch.empty(R, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    _, mean, rstd = ctx.layer_norm(x, stats=True)
    _, dw, db = ctx.layer_norm_grad(dy, x, torch.ones(d, device=DEV), mean, rstd)
    ctx.sync()
    want = torch.zeros(2, d, dtype=torch.float64, device=DEV)
    mag = torch.zeros(2, d, dtype=torch.float64, device=DEV)
    for a in range(0, R, 1 << 17):
        at = slice(a, a + (1 << 17))
        n = (x[at].double() - mean[at].double()[:, None]) * rstd[at].double()[:, None]
        y = dy[at].double()
        for k, terms in enumerate((y * n, y)):
            want[k] += terms.sum(0)
            mag[k] += terms.abs().sum(0)
    for k, got in enumerate((dw, db)):
        assert ((got.double() - want[k]).abs() <= 4096 * U * mag[k]).all()


def test_reserve_for_more_columns_than_a_call_takes(sph, ctx):
    x, dy = rows_of(1, 300, torch.float32, 1), rows_of(1, 300, torch.float32, 2)
    w, _ = params(300, torch.float32, 3)
    _, mean, rstd = ctx.layer_norm(x, w, stats=True)
    want = ctx.layer_norm_grad(dy, x, w, mean, rstd)
    own = sph.Context(0)
    own.reserve(1, 1, 1 << 31)
    own.reserve(1, 1, (1 << 31) + 4096)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = own.layer_norm_grad(dy, x, w, mean, rstd)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    own.close()


def test_other_streams_and_graphs(sph, ctx):
    R, d = 333, 1500
    x, dy = rows_of(R, d, torch.bfloat16, 1), rows_of(R, d, torch.bfloat16, 2)
    w, b = params(d, torch.float32, 3)
    want = ctx.layer_norm(x, w, b, stats=True)
    wantg = ctx.layer_norm_grad(dy, x, w, want[1], want[2])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = ctx.layer_norm(x, w, b, stats=True)
        gotg = ctx.layer_norm_grad(dy, x, w, got[1], got[2])
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want + wantg, got + gotg))
    own = sph.Context(0)
    own.reserve(R, 1, d)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = own.layer_norm(x, w, b, stats=True)
        gotg = own.layer_norm_grad(dy, x, w, got[1], got[2])
    for seed in (1, 7):
        x.copy_(rows_of(R, d, torch.bfloat16, seed))
        g.replay()
        torch.cuda.synchronize()
        ref = ctx.layer_norm(x, w, b, stats=True)
        refg = ctx.layer_norm_grad(dy, x, w, ref[1], ref[2])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref + refg, got + gotg))
    own.close()


def test_profile_counts_the_calls(sph, ctx):
    x = rows_of(3, 64, torch.float32, 1)
    ctx.profile_enable(True)
    _, mean, rstd = ctx.layer_norm(x, stats=True)
    ctx.layer_norm_grad(x, x, None, mean, rstd)
    p = ctx.profile_read()
    ctx.profile_enable(False)
    assert p["calls"]["rows"] == 2 and p["launches"] == 3


def test_refusals(sph, ctx):
    x = rows_of(4, 64, torch.float32, 1)
    w, b = params(64, torch.float32, 2)
    _, mean, rstd = ctx.layer_norm(x, stats=True)
    bad = [lambda: ctx.layer_norm(x.double()), lambda: ctx.layer_norm(x[0]),
           lambda: ctx.layer_norm(x.t()), lambda: ctx.layer_norm(x, w[:63]),
           lambda: ctx.layer_norm(x, w, b.half()), lambda: ctx.layer_norm(x, w[::2]),
           lambda: ctx.layer_norm(x, w.cpu()), lambda: ctx.layer_norm(x, out=x[:3]),
           lambda: ctx.layer_norm(x, dtype=torch.int32),
           lambda: ctx.layer_norm_grad(x, x[:3], w, mean, rstd),
           lambda: ctx.layer_norm_grad(x, x, w, mean[:3], rstd),
           lambda: ctx.layer_norm_grad(x, x, w, mean, rstd.double()),
           lambda: ctx.layer_norm_grad(x, x, w, mean, rstd, accumulate=True),
           lambda: ctx.layer_norm_grad(x, x, w, mean, rstd, d_weight=torch.empty(63, device=DEV)),
           lambda: ctx.layer_norm_grad(x, x, w, mean, rstd, d_x=x[:, :63])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ctx.layer_norm(x, eps=-1.0), lambda: ctx.layer_norm(x, eps=float("nan")),
                 lambda: ctx.layer_norm(x, eps=float("inf")),
                 lambda: ctx.layer_norm_grad(x, x, w, mean, None)):
        with pytest.raises(sph.SphError):
            call()
    assert sph.lib.sph_layer_norm(ctx.handle, x.data_ptr(), 1, 4, 64, 63, None, None, 1, 1e-5, 1,
                                  x.data_ptr(), 1, 64, None, None) == 1
    assert sph.lib.sph_layer_norm(ctx.handle, x.data_ptr(), 1, 1, (1 << 20) + 1, 1 << 21, None, None,
                                  1, 1e-5, 1, x.data_ptr(), 1, 1 << 21, None, None) == 2
    check_y(ctx.layer_norm(x, w, b), x, w, b, True, 1e-5, torch.float32)
