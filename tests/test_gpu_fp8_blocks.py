"""Rows in e4m3 with a scale for each block of 128 columns, and the product with a table held
so, against the 64-bit oracle.

Tolerances, from the arithmetic (u = 2^-24):
  quantise   codes and scales are decided by exact comparisons: equal
  values     one rounding to fp32, one to the output's type
  product    the terms are exact products of 4-bit significands; an MMA adds 32 of them and
             what it holds, aligned to the largest, none losing more than 2^-23 of that: four
             MMAs a block, 4 * 33 * 2 u of the sum of magnitudes; then two roundings a block's
             sum and one an addition over the blocks, and the scales' product's own
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import rows_oracle as ora  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
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
    return t.detach().double().cpu().numpy()


def make_x(rows, d, dtype, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, d)) * np.exp(rng.standard_normal((rows, 1)))
    x[:, ::37] *= 30
    x[:, 130:140] *= 1e-3
    return torch.tensor(x, dtype=torch.float32).to(dtype).to(DEV)


def bytes_of(w):
    return w.codes.view(torch.uint8).cpu().numpy()


def same_floats(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])


# ---- quantise -------------------------------------------------------------------
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 15), (2, 127), (5, 128), (130, 129), (1, 512),
                                    (300, 513), (129, 1000), (7, 4097)])
def test_quantise_equals_the_oracle(sph, ctx, block, dtype, rows, d):
    x = make_x(rows, d, dtype, rows + d)
    w = ctx.fp8_quantize(x, block)
    back = {t: ctx.fp8_dequantize(w, dtype=t) for t in TYPES}
    ctx.sync()
    codes, scales = ora.encode8(f64(x), block)
    assert w.codes.dtype == torch.float8_e4m3fn and w.block_rows == block
    assert np.array_equal(f64(w.scales), scales.astype(np.float64))
    assert np.array_equal(bytes_of(w), codes)
    want = ora.decode8(codes, scales, block)
    for t in TYPES:
        off = np.abs(f64(back[t]) - want)
        with np.errstate(invalid="ignore"):
            ok = off <= (U + HALF[t]) * np.abs(want) * 1.01 + 2.0 ** -25
        assert (ok | (np.abs(want) > 65000)).all()
    assert np.abs(f64(back[torch.float32]) - f64(x)).max() <= 2.0 ** -4 * np.abs(f64(x)).max()


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -100, 2.0 ** 100, 3.7e-12, 1.1e19])
def test_borders_of_two_codes(sph, ctx, block, scale):
    # values on the borders of two codes, and beside them by a step, in units of scales that
    # are no powers of two: where a rounded quotient would land on the border itself
    grid = ora._E4M3
    rng = np.random.default_rng(3)
    x = np.zeros((256, 128), np.float32)
    for r in range(256):
        top = np.float32(448 * scale * (1 + rng.random()))
        s = np.float32(top / np.float32(448))
        mids = (grid[1:] + grid[:-1]) / 2
        v = np.float32(rng.permutation(mids)[:126] * np.float64(s))
        v = np.nextafter(v, np.float32(np.where(rng.random(126) < 0.5, np.inf, -np.inf)),
                         dtype=np.float32) if r % 3 == 1 else v
        x[r, 0], x[r, 1:127] = top, v * np.where(rng.random(126) < 0.5, -1, 1)
    if block == 128:
        x[:128, 0], x[128:, 0] = x[0, 0], x[255, 0]
        for r in range(256):
            s = np.float64(np.float32(x[r, 0] / np.float32(448)))
            x[r, 1:127] = np.float32(np.random.default_rng(r).permutation((grid[1:] + grid[:-1]) / 2) * s)
    w = ctx.fp8_quantize(torch.tensor(x, device=DEV), block)
    ctx.sync()
    codes, scales = ora.encode8(x, block)
    assert np.array_equal(f64(w.scales), scales.astype(np.float64))
    assert np.array_equal(bytes_of(w), codes)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_borders_in_16_bits(sph, ctx, dtype):
    # every magnitude of a type against a largest one that is a multiple of 7: exact quotients
    # on the borders of two codes
    bits = np.arange(1, 1 << 15, dtype=np.int16)
    vals = torch.tensor(bits).view(dtype)
    vals = vals[torch.isfinite(vals.float())]
    for top in (7.0, 448.0, 3.5, 1.0, 0.0546875):
        x = vals[vals.float() <= top]
        x = torch.cat([x, torch.zeros(-len(x) % 127, dtype=dtype)]).view(-1, 127)
        x = torch.cat([torch.full((len(x), 1), top, dtype=dtype), x], 1).to(DEV)
        w = ctx.fp8_quantize(x)
        ctx.sync()
        codes, scales = ora.encode8(f64(x))
        assert np.array_equal(f64(w.scales), scales.astype(np.float64))
        assert np.array_equal(bytes_of(w), codes)


@pytest.mark.parametrize("dtype,bits,power", [
    (torch.bfloat16, 8, 0), (torch.bfloat16, 8, -127), (torch.bfloat16, 8, -118), (torch.bfloat16, 8, -69),
    (torch.bfloat16, 8, 120), (torch.float16, 11, -6), (torch.float16, 11, -20), (torch.float16, 11, 4)])
@pytest.mark.parametrize("block", [1, 128])
def test_every_pair_of_mantissas(sph, ctx, dtype, bits, power, block):
    # (scales at and next to the least one, and from subnormal magnitudes, too)
    # quotients half way between two codes but for what rounding the scale took, and those that
    # are exact: every significand of x under every (fp16: every 17th) significand of amax
    half = 1 << bits - 1
    amax = torch.arange(half, 2 * half, 1 if bits == 8 else 17, dtype=torch.float64)
    low = 20 if bits == 8 else 3
    x = torch.cat([torch.arange(half, 2 * half, dtype=torch.float64) * 2.0 ** -e
                   for e in range(1, low)])
    if block == 1:
        x = torch.cat([x, torch.zeros(-len(x) % 127, dtype=torch.float64)]).reshape(-1, 127)
        x[:, ::2] *= -1
        rows = torch.cat([amax[:, None, None].expand(-1, len(x), 1),
                          x[None].expand(len(amax), -1, -1)], 2).reshape(len(amax), -1)
    else:
        rows = torch.zeros(len(amax), 128 * 128, dtype=torch.float64)
        rows[:, :len(x)] = x
        rows[:, ::2] *= -1
        rows[:, -1] = amax
        rows = rows.reshape(-1, 128)
    rows = (rows * 2.0 ** power).to(dtype).to(DEV)
    w = ctx.fp8_quantize(rows, block)
    ctx.sync()
    codes, scales = ora.encode8(f64(rows), block)
    assert np.array_equal(f64(w.scales), scales.astype(np.float64))
    assert np.array_equal(bytes_of(w), codes)


@pytest.mark.parametrize("block", [1, 128])
def test_quantise_extremes(sph, ctx, block):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((8 * block, 300)).astype(np.float32)
    for i in range(8):
        at = slice(i * block, (i + 1) * block)
        if i == 0: x[at] = 0
        if i == 1: x[at] *= np.float32(1e-38)
        if i == 2: x[at] = 1e-42                      # subnormal
        if i == 3: x[at] *= np.float32(5e37)
        if i == 4: x[i * block, 140] = np.inf
        if i == 5: x[i * block, 3], x[(i + 1) * block - 1, 290] = np.nan, -np.inf
        if i == 6: x[at, :150] *= np.float32(1e-12)
        if i == 7: x[at] = -0.0
    w = ctx.fp8_quantize(torch.tensor(x, device=DEV), block)
    back = ctx.fp8_dequantize(w, dtype=torch.float32)
    ctx.sync()
    codes, scales = ora.encode8(x, block)
    assert same_floats(f64(w.scales), scales) and np.array_equal(bytes_of(w), codes)
    want = ora.decode8(codes, scales, block)
    got = f64(back)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert (np.abs(got[ok] - want[ok]) <= U * np.abs(want[ok]) + 2.0 ** -150).all()


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("off", [0, 1, 3, 8])
def test_quantise_strided_rows_and_given_buffers(sph, ctx, block, off):
    x = make_x(262, 400, torch.bfloat16, 11)[::2, off:off + 211]
    codes = torch.full((262, 240), 0xEE, dtype=torch.uint8, device=DEV)
    scales = torch.full((131, 4), 9.0, device=DEV)
    out = sph.Fp8(codes[::2, :211], scales[:131 if block == 1 else 2, :2], block)
    assert ctx.fp8_quantize(x, block, out=out) is out
    ctx.sync()
    want, ws = ora.encode8(f64(x), block)
    assert np.array_equal(bytes_of(out), want) and np.array_equal(f64(out.scales), ws.astype(np.float64))
    assert (codes[:, 211:] == 0xEE).all() and (codes[1::2] == 0xEE).all() and (scales[:, 2:] == 9).all()


# ---- lookup ----------------------------------------------------------------------
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("d", [1, 100, 513, 2000])
@pytest.mark.parametrize("out", TYPES)
def test_lookup(sph, ctx, block, d, out):
    V = 200
    w = ctx.fp8_quantize(make_x(V, d, torch.float32, d), block)
    table = ora.decode8(bytes_of(w), w.scales.cpu().numpy(), block)
    tok = torch.tensor([0, 199, 5, -1, 5, 7, 130], dtype=torch.int32, device=DEV)
    wide = torch.full((7, d + 3), 5.0, dtype=out, device=DEV)
    for dst in (None, wide[:, 1:d + 1]):
        y = ctx.embed(tok, w, scale=3.0, padding_id=7, dtype=out, out=dst)
        torch.cuda.synchronize()
        want = np.where(np.isin(tok.cpu().numpy(), (-1, 7))[:, None], 0, 3.0 * table[tok.cpu().numpy()])
        assert (np.abs(f64(y) - want) <= (2 * U + HALF[out]) * np.abs(want) * 1.01 + 2.0 ** -25).all()
    assert (wide[:, 0] == 5).all() and (wide[:, d + 1:] == 5).all()
    with pytest.raises(sph.SphError):      # the token outside the table
        ctx.sync()
    ctx.sync()
    assert ctx.embed(tok[:0], w).shape == (0, d)


# ---- product ---------------------------------------------------------------------
def check(y, h, table, ids=None, bias=None, out=torch.float32):
    want, mag = ora.product8(f64(h), table, None if ids is None else ids.cpu().numpy(),
                             None if bias is None else f64(bias))
    blocks = -(-h.shape[1] // 128)
    bound = (4 * 33 * 2 + blocks + 6) * U * mag + (U + HALF[out] * 1.01) * np.abs(want)
    assert (np.abs(f64(y) - want) <= bound).all()
    return want


def held(ctx, V, d, block, seed):
    w = ctx.fp8_quantize(make_x(V, d, torch.float32, seed), block)
    return w, ora.decode8(bytes_of(w), w.scales.cpu().numpy(), block)


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,V,d", [(1, 128, 128), (1, 2, 1), (3, 130, 33), (16, 300, 256),
                                      (17, 257, 300), (33, 140, 129), (65, 500, 1025), (130, 260, 640),
                                      (200, 129, 500)])
def test_product_whole_vocabulary(sph, ctx, block, rows, V, d):
    w, table = held(ctx, V, d, block, V + d)
    for ht in (torch.float32, torch.bfloat16):
        h = make_x(rows, d, ht, rows)
        y = ctx.fp8_logits(h, w)
        ctx.sync()
        check(y, h, table)


def subset(kind, V, rng):
    return {"runs": np.concatenate([np.arange(5, 140), np.arange(200, 264), np.arange(500, 700)]),
            "odd": np.arange(1, V, 2), "single": np.array([V - 1]),
            "mixed": np.concatenate([np.arange(64), np.sort(rng.choice(np.arange(70, 690), 177, False))]),
            "all": np.arange(V)}[kind]


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows", [2, 31, 129, 260])
@pytest.mark.parametrize("kind", ["runs", "odd", "single", "mixed", "all"])
@pytest.mark.parametrize("pair", [0, 1, 2])
def test_product_of_kept_rows(sph, ctx, block, rows, kind, pair):
    V, d = 700, 200
    rng = np.random.default_rng(rows)
    ids = torch.tensor(subset(kind, V, rng).astype(np.int32), device=DEV)
    w, table = held(ctx, V, d, block, 4)
    h = make_x(rows, d + 3, torch.float32, rows)[:, 3:]
    bias = torch.tensor(rng.standard_normal(V), dtype=torch.float32, device=DEV)
    n = ids.numel()
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_TC_PAIR, pair)
    for out in (torch.float32, torch.bfloat16):
        wide = torch.full((rows, n + 5), 3.0, dtype=out, device=DEV)
        y = c.fp8_logits(h, w, keep_ids=ids, bias=bias, out=wide[:, 2:n + 2])
        c.sync()
        check(y, h, table, ids, bias, out)
        assert (wide[:, :2] == 3).all() and (wide[:, n + 2:] == 3).all()
    c.close()


@pytest.mark.parametrize("pair", [0, 1, 2])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,V,d", [(16, 30000, 384), (100, 40000, 200), (200, 30000, 256),
                                      (500, 9000, 300)])
def test_many_tiles(sph, ctx, pair, block, rows, V, d):
    # several tiles a CTA: every logit against the 64-bit product of what the device holds
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_TC_PAIR, pair)
    g = torch.Generator(device=DEV).manual_seed(rows + block)
    w = c.fp8_quantize(torch.randn(V, d, generator=g, device=DEV) * 0.02, block)
    h = torch.randn(rows, d, generator=g, device=DEV)
    y = c.fp8_logits(h, w)
    c.sync()
    hq = c.fp8_quantize(h)
    values = lambda q: q.codes.double() * q.scales.double().repeat_interleave(128, 1)[:, :d] \
        .repeat_interleave(q.block_rows, 0)[:q.codes.shape[0]]
    x, t = values(hq), values(w)
    want, mag = x @ t.T, x.abs() @ t.abs().T
    off = (y.double() - want).abs()
    assert (off <= (4 * 33 * 2 + 9) * U * mag + U * want.abs()).all()
    assert float(off.norm() / want.norm()) < 2e-6
    c.close()


@pytest.mark.parametrize("pair", [1, 2])
@pytest.mark.parametrize("block,rows", [(1, 40), (128, 40), (128, 130)])
def test_scales_far_apart(sph, ctx, pair, block, rows):
    # a logit is finite wherever its products' magnitudes add up within range
    V, d = 1500, 260
    rng = np.random.default_rng(0)
    exps = np.repeat(rng.integers(-116, 110, -(-V // block)), block)[:V, None]
    table = (rng.standard_normal((V, d)) * 2.0 ** exps.astype(np.float64)).astype(np.float32)
    table[7] = 0
    hid = rng.standard_normal((rows, d)).astype(np.float32)
    exps = rng.integers(-100, 100, rows)
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_TC_PAIR, pair)
    w = c.fp8_quantize(torch.tensor(table, device=DEV), block)
    h = torch.tensor(hid * (2.0 ** exps.astype(np.float64))[:, None], dtype=torch.float32, device=DEV)
    y = f64(c.fp8_logits(h, w))
    c.sync()
    want, mag = ora.product8(f64(h), ora.decode8(bytes_of(w), w.scales.cpu().numpy(), block))
    inside = mag < 2.0 ** 127
    assert inside.any() and not inside.all()
    off = np.abs(y[inside] - want[inside])
    assert (off <= (4 * 33 * 2 + 9) * U * mag[inside] + U * np.abs(want[inside]) + 8 * 2.0 ** -149).all()
    assert (y[:, 7] == 0).all()
    c.close()


def test_nan_blocks_stay_in_their_rows_and_ids(sph, ctx):
    x, t = make_x(5, 300, torch.float32, 1), make_x(200, 300, torch.float32, 2)
    x[3, 200], t[150, 5] = float("inf"), float("nan")
    w = ctx.fp8_quantize(t)
    y = ctx.fp8_logits(x, w)
    ctx.sync()
    bad = torch.zeros(5, 200, dtype=torch.bool, device=DEV)
    bad[3], bad[:, 150] = True, True
    assert torch.equal(y.isnan(), bad)


@pytest.mark.parametrize("pair", [0, 1, 2])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("block,rows", [(1, 5), (1, 40), (1, 100), (1, 260), (128, 5), (128, 40),
                                        (128, 130), (128, 260)])
def test_bad_hidden_states_beside_zero_rows(sph, pair, kept, block, rows):
    # a NaN or an infinity of a hidden state reaches each of its logits, and no other's, whatever
    # the table's scales and the number of rows: those of zeros have 2^-126
    V, d = 700, 300
    table = make_x(V, d, torch.float32, 7)
    table[7], table[256:384] = 0, 0
    h = make_x(rows, d, torch.float32, rows)
    h[1, 70], h[3, 299], h[rows - 1, 0], h[2] = float("nan"), float("inf"), float("-inf"), 0
    bad = torch.tensor(sorted({1, 3, rows - 1}), device=DEV)
    good = torch.tensor([r for r in range(rows) if r not in (1, 3, rows - 1)], device=DEV)
    ids = np.concatenate([np.arange(100), np.arange(101, 300, 2), np.arange(350, 390), [600]])
    ids = torch.tensor(ids.astype(np.int32), device=DEV) if kept else None
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_TC_PAIR, pair)
    w = c.fp8_quantize(table, block)
    y = c.fp8_logits(h, w, keep_ids=ids)
    c.sync()
    assert y[bad].isnan().all()
    check(y[good], h[good], ora.decode8(bytes_of(w), w.scales.cpu().numpy(), block), ids)
    c.close()


def test_a_wait_that_gives_up(sph, ctx):
    c = sph.Context(0)
    for pair, block, rows in ((2, 1, 9), (1, 1, 9), (0, 128, 90)):
        w, table = held(ctx, 300, 200, block, 4)
        h = make_x(rows, 200, torch.float32, 1)
        ctx.sync()
        c.set_option(sph.SPH_OPT_TC_PAIR, pair)
        c.set_option(sph.SPH_OPT_SPIN_LIMIT, 1)
        c.fp8_logits(h, w)
        with pytest.raises(sph.SphError) as e:
            c.sync()
        assert e.value.status == 4
        c.set_option(sph.SPH_OPT_SPIN_LIMIT, 1 << 34)
        y = c.fp8_logits(h, w)
        c.sync()
        check(y, h, table)
    c.close()


@pytest.mark.parametrize("pair,rows", [(1, 230), (2, 130)])
@pytest.mark.parametrize("kept", [False, True])
def test_a_wait_that_gives_up_with_many_hidden_states(sph, pair, rows, kept):
    # hidden states as the MMA's M, and the tiles of scales far from 1 after them
    V, d = 900, 1000
    table = make_x(V, d, torch.float32, 3)
    table[256:384] = 0
    h = make_x(rows, d, torch.float32, 1)
    ids = torch.tensor([i for i in range(V) if i % 5 or i < 300], dtype=torch.int32, device=DEV) if kept else None
    c = sph.Context(0)
    w = c.fp8_quantize(table, 128)
    c.sync()
    c.set_option(sph.SPH_OPT_TC_PAIR, pair)
    for _ in range(2):
        c.set_option(sph.SPH_OPT_SPIN_LIMIT, 1)
        c.fp8_logits(h, w, keep_ids=ids)
        with pytest.raises(sph.SphError) as e:
            c.sync()
        assert e.value.status == 4
        c.set_option(sph.SPH_OPT_SPIN_LIMIT, 1 << 34)
        y = c.fp8_logits(h, w, keep_ids=ids)
        c.sync()
        check(y, h, ora.decode8(bytes_of(w), w.scales.cpu().numpy(), 128), ids)
    c.close()


def test_streams_graphs_and_reserve(sph, ctx):
    V, d, rows = 500, 300, 20
    w, table = held(ctx, V, d, 128, 4)
    ids = torch.arange(0, V, 3, dtype=torch.int32, device=DEV)
    h = make_x(rows, d, torch.float32, 1)
    want = ctx.fp8_logits(h, w, keep_ids=ids)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = ctx.fp8_logits(h, w, keep_ids=ids)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    own = sph.Context(0)
    own.reserve(rows, V, d)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q = own.fp8_quantize(h)
        got = own.fp8_logits(h, w, keep_ids=ids)
        back = own.fp8_dequantize(q, dtype=torch.float32)
    for seed in (2, 3):
        h.copy_(make_x(rows, d, torch.float32, seed))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, ctx.fp8_logits(h, w, keep_ids=ids))
        assert torch.equal(back, ctx.fp8_dequantize(ctx.fp8_quantize(h), dtype=torch.float32))
    own.close()


def test_far_table(sph, ctx):
    # codes past 2^31 bytes
    V, d = 530000, 4112
    codes = torch.zeros(V, d, dtype=torch.uint8, device=DEV)
    scales = torch.ones(V, 33, device=DEV)
    far = [0, 1, V - 130, V - 2, V - 1]
    x = make_x(len(far), d, torch.float32, 1)
    q = ctx.fp8_quantize(x)
    ctx.sync()
    for i, r in enumerate(far):
        codes[r], scales[r] = q.codes.view(torch.uint8)[i], q.scales[i]
    w = sph.Fp8(codes, scales, 1)
    ids = torch.tensor(far, dtype=torch.int32, device=DEV)
    h = make_x(3, d, torch.float32, 5)
    y = ctx.fp8_logits(h, w, keep_ids=ids)
    full = ctx.fp8_logits(h, w)
    rows = ctx.embed(ids, w, dtype=torch.float32)
    ctx.sync()
    check(y, h, ora.decode8(bytes_of(q), q.scales.cpu().numpy()))
    assert torch.equal(full[:, ids.long()], y) and (full[:, 2:V - 130] == 0).all()
    assert torch.equal(rows, ctx.fp8_dequantize(q, dtype=torch.float32))


def test_one_row_tables_and_odd_scale_strides(sph, ctx):
    t = make_x(1, 300, torch.float32, 1)
    w = ctx.fp8_quantize(t, 128)
    h = make_x(2, 300, torch.float32, 2)
    table = ora.decode8(bytes_of(w), w.scales.cpu().numpy(), 128)
    one = sph.Fp8(w.codes.clone(), w.scales.clone(), 1)
    for q in (w, one):
        y = ctx.fp8_logits(h, q)
        ctx.sync()
        check(y, h, table)
    w, table = held(ctx, 260, 300, 1, 3)
    odd = torch.zeros(260, 7, device=DEV)
    odd[:, 2:5] = w.scales
    y = ctx.fp8_logits(h, sph.Fp8(w.codes, odd[:, 2:5], 1))
    ctx.sync()
    check(y, h, table)


def test_refusals(sph, ctx):
    w, _ = held(ctx, 200, 300, 1, 1)
    w128, _ = held(ctx, 200, 300, 128, 1)
    h = make_x(4, 300, torch.float32, 2)
    narrow = torch.zeros(200, 310, dtype=torch.uint8, device=DEV)[:, :300]
    bad = [lambda: ctx.fp8_quantize(h, 64), lambda: ctx.fp8_quantize(h.double()),
           lambda: ctx.fp8_quantize(h, 1, out=w), lambda: ctx.fp8_quantize(h, 128, out=w),
           lambda: ctx.fp8_logits(h[:, :299], w), lambda: ctx.fp8_logits(h, sph.Fp8(w.codes, w.scales, 128)),
           lambda: ctx.fp8_logits(h, sph.Fp8(w128.codes, w128.scales, 1)),
           lambda: ctx.fp8_logits(h, sph.Fp8(w.codes, w.scales.double(), 1)),
           lambda: ctx.fp8_logits(h, sph.Fp8(w.codes.cpu(), w.scales, 1)),
           lambda: ctx.fp8_logits(h, w, bias=torch.zeros(199, device=DEV)),
           lambda: ctx.fp8_logits(h, w, keep_ids=torch.arange(3, device=DEV)),
           lambda: ctx.fp8_logits(h, w, out=torch.empty(4, 199, device=DEV)),
           lambda: sph.fp8_empty(3, 4, 2), lambda: sph.fp8_empty(0, 4)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ctx.fp8_logits(h, w, dtype=torch.float16),
                 lambda: ctx.fp8_logits(h, sph.Fp8(narrow, w.scales, 1)),
                 lambda: ctx.fp8_logits(h[:0], w)):
        with pytest.raises(sph.SphError):
            call()
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_CHECK_IDS, 1)
    for ids in ([3, 3], [5, 4], [0, 200], [-1, 2]):
        with pytest.raises(sph.SphError):
            c.fp8_logits(h, w, keep_ids=torch.tensor(ids, dtype=torch.int32, device=DEV))
    c.close()
