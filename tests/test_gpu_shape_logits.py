"""Logits with penalties, biases and masks, and tokens from them.

The definition's steps are single fp32 operations, so results equal the same steps in fp32
(numpy's), bit by bit, and lie within six roundings of the magnitudes of the 64-bit ones.
A greedy token is the first largest of the written logits.  A drawn one lies where the 64-bit
cumulated probabilities pass the uniform, to within 1e-5: an id's weight is off by the
exponential's 2^-22 and the argument's two roundings (|z - max| / tau <= 100 of them weighted
by exp(-|z - max| / tau): below 2^-23 together), sums by at most 64 additions in turn.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import oracle  # noqa: E402
from oracle import rows_oracle as ora  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
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


def dev(a, dtype):
    return torch.tensor(np.asarray(a), dtype=dtype).to(DEV)


def make(R, n, V, seed, ids=None, tokens=40, biases=5, mask=0.6, mask_rows=None):
    """Arguments in numpy, of all kinds."""
    rng = np.random.default_rng(seed)
    a = dict(ids=ids)
    if tokens:
        h = rng.integers(-3, V + 3, (R, tokens))
        h[:, ::3] = rng.integers(0, min(V, 12), h[:, ::3].shape)        # (repeated ones)
        a.update(history=h, lengths=rng.integers(0, tokens + 1, R), prompts=rng.integers(0, tokens + 1, R),
                 repetition=np.float32(rng.uniform(0.5, 2, R)), frequency=np.float32(rng.uniform(-1, 1, R)),
                 presence=np.float32(rng.uniform(-1, 1, R)))
    if biases:
        b = rng.integers(-2, V + 2, (R, biases))
        b[:, biases // 2:] = b[:, :biases - biases // 2]                # (the same id twice)
        a.update(bias_ids=b, bias_values=np.float32(rng.standard_normal((R, biases)) * 3))
    if mask:
        M = R if mask_rows is None else 3
        words = np.zeros((M, -(-V // 32)), np.uint32)
        bits = rng.random((M, words.shape[1] * 32)) < mask
        for j in range(32):
            words |= bits[:, j::32].astype(np.uint32) << np.uint32(j)
        a["mask"] = words.astype(np.int64) - (words >= 2 ** 31).astype(np.int64) * 2 ** 32
        if mask_rows is not None:
            a["mask_rows"] = rng.integers(-1, M, R)
    return np.float32(rng.standard_normal((R, n)) * 4), a


def call(ctx, z, V, a, **kw):
    g = lambda k, t: None if a.get(k) is None else dev(a[k], t)
    i, f = torch.int32, torch.float32
    return ctx.shape_logits(z, V, keep_ids=g("ids", i), history=g("history", i),
                            lengths=g("lengths", i), prompt_lengths=g("prompts", i),
                            repetition=g("repetition", f), frequency=g("frequency", f),
                            presence=g("presence", f), bias_ids=g("bias_ids", i),
                            bias_values=g("bias_values", f), mask=g("mask", i),
                            mask_rows=g("mask_rows", i), **kw)


def first_largest(y, ids):
    out = []
    for row in y:
        j = int(row.argmax())
        out.append(-1 if row[j] == -np.inf else j if ids is None else int(ids[j]))
    return out


def same(a, b):
    return np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])


SIZES = [(1, 1), (2, 7), (3, 31), (1, 32), (2, 33), (5, 100), (3, 2047), (2, 2048), (2, 2049),
         (1, 4103), (700, 130), (40, 9000), (2, 40000)]


@pytest.mark.parametrize("R,n", SIZES)
@pytest.mark.parametrize("kept", [False, True])
def test_every_step_in_fp32(ctx, R, n, kept):
    V = n if not kept else 2 * n + 5
    ids = None if not kept else np.sort(np.random.default_rng(n).choice(V, n, False))
    z, a = make(R, n, V, n + R, ids)
    y, t = call(ctx, dev(z, torch.float32), V, a, temperature=0.0)
    ctx.sync()
    want = ora.shape(z, V, **a, dtype=np.float32)
    assert same(y.cpu().numpy(), want)
    assert t.tolist() == first_largest(want, ids)
    with np.errstate(invalid="ignore"):
        exact = ora.shape(z, V, **a)
        size = 2 * np.abs(z) + 2 * 40 + 60
        assert (np.abs(want - exact)[np.isfinite(exact)] <= (6 * 2.0 ** -24 * size)[np.isfinite(exact)]).all()


@pytest.mark.parametrize("zt", TYPES)
@pytest.mark.parametrize("ot", TYPES)
@pytest.mark.parametrize("off", [0, 1, 2])
def test_types_strides_and_alignments(ctx, zt, ot, off):
    R, n, V = 5, 2500, 2500
    z, a = make(R, n, V, 3)
    zd = torch.zeros(R, n + 8, dtype=zt, device=DEV)
    zd[:, off:off + n] = dev(z, torch.float32).to(zt)
    out = torch.full((2 * R, n + 9), 7.0, dtype=ot, device=DEV)
    y = call(ctx, zd[:, off:off + n], V, a, out=out[::2, off:off + n])
    ctx.sync()
    want = ora.shape(zd[:, off:off + n].float().cpu().numpy(), V, **a, dtype=np.float32)
    assert same(y.float().cpu().numpy(), torch.tensor(want).to(ot).float().numpy())
    assert (out[1::2] == 7).all() and (out[:, off + n:] == 7).all() and (out[:, :off] == 7).all()


@pytest.mark.parametrize("what", [("tokens",), ("biases",), ("mask",), ()])
@pytest.mark.parametrize("n", [50, 5000])
def test_each_alone_and_none(ctx, what, n):
    kw = dict(tokens=0, biases=0, mask=0)
    if "tokens" in what: kw["tokens"] = 30
    if "biases" in what: kw["biases"] = 70
    if "mask" in what: kw["mask"] = 0.3
    z, a = make(4, n, n, 5, **kw)
    want = ora.shape(z, n, **a, dtype=np.float32)
    y = call(ctx, dev(z, torch.float32), n, a)
    assert same(y.cpu().numpy(), want)
    for drop in ("lengths", "prompts", "repetition", "frequency", "presence"):
        if drop in a:
            b = {k: v for k, v in a.items() if k != drop}
            y = call(ctx, dev(z, torch.float32), n, b)
            assert same(y.cpu().numpy(), ora.shape(z, n, **b, dtype=np.float32))


def test_in_place_needs_the_same_form(sph, ctx):
    z = torch.randn(4, 64, device=DEV)
    was = z.clone()
    for call in (lambda: ctx.shape_logits(z, 64, out=z.view(torch.bfloat16)[:, :64]),
                 lambda: ctx.shape_logits(z[:2], 64, out=z[::2])):
        with pytest.raises(sph.SphError):
            call()
    ctx.sync()
    assert torch.equal(z, was)


def test_masks_by_index_and_in_place(ctx):
    z, a = make(9, 3000, 3000, 7, mask_rows=True)
    zd = dev(z, torch.float32)
    want = ora.shape(z, 3000, **a, dtype=np.float32)
    y, t = call(ctx, zd, 3000, a, out=zd, temperature=0.0)
    ctx.sync()
    assert y is zd and same(y.cpu().numpy(), want) and t.tolist() == first_largest(want, None)


def test_a_mask_out_of_range_is_reported(sph, ctx):
    z, a = make(4, 100, 100, 7, mask_rows=True)
    a["mask_rows"] = np.array([0, 3, -1, -2])
    y = call(ctx, dev(z, torch.float32), 100, a)
    torch.cuda.synchronize()
    a["mask_rows"] = np.array([0, -1, -1, -1])
    assert same(y.cpu().numpy(), ora.shape(z, 100, **a, dtype=np.float32))
    with pytest.raises(sph.SphError):
        ctx.sync()
    ctx.sync()


@pytest.mark.parametrize("n", [5, 3000, 9000])
@pytest.mark.parametrize("temperature", [0.0, 0.7])
def test_empty_rows_nan_and_infinity(ctx, n, temperature):
    z = np.float32(np.random.default_rng(1).standard_normal((8, n)))
    mask = np.full((8, -(-n // 32)), -1, np.int64)
    mask[0] = 0                                   # nothing is allowed
    z[1] = -np.inf                                # nothing is left
    z[2, n - 1] = np.nan                          # an allowed NaN
    z[3, 2], z[3, 1] = np.nan, -np.inf            # a masked NaN
    mask[3, 0] = -1 - (1 << 2)
    z[4, 3] = np.inf                              # drawn for certain
    z[5], z[5, 4] = -np.inf, -3e38                # one id left
    z[6, 1] = np.inf                              # masked
    mask[6, 0] = -1 - (1 << 1)
    z[7] = np.float32(-1e30)                      # all alike
    y, t = call(ctx, dev(z, torch.float32), n, dict(mask=mask), temperature=temperature, seed=3)
    ctx.sync()
    want = ora.shape(z, n, mask=mask, dtype=np.float32)
    assert same(y.cpu().numpy(), want)
    t = t.tolist()
    assert t[0] == t[1] == t[2] == -1 and t[4] == 3 and t[5] == 4 and t[6] not in (-1, 1)
    assert t[3] not in (-1, 1, 2) and 0 <= t[7] < n
    if temperature == 0:
        assert t[7] == 0 and t[3] == int(np.nanargmax(want[3]))


def test_ties_go_to_the_lowest_id(ctx):
    for n in (40, 5000, 20000):
        z = np.zeros((4, n), np.float32)
        z[1, n // 2:] = 1
        z[2, [n - 1, 3]] = 2
        z[3, n - 1] = 5
        ids = np.arange(n) * 2 + 1
        _, t = call(ctx, dev(z, torch.float32), 2 * n + 1, dict(ids=ids), temperature=0.0)
        assert t.tolist() == [1, 2 * (n // 2) + 1, 7, 2 * n - 1]


@pytest.mark.parametrize("n", [1, 40, 2049, 30000])
@pytest.mark.parametrize("temperature", [0.3, 1.0, 3.0])
@pytest.mark.parametrize("aligned", [True, False])
def test_draws(ctx, n, temperature, aligned):
    R = 64
    z, a = make(R, n, n, n, tokens=20, biases=3, mask=0.5)
    out = torch.empty(R, n if aligned else n + 1, device=DEV)[:, :n]
    y, t = call(ctx, dev(z, torch.float32), n, a, temperature=temperature, seed=11, offset=1 << 33, out=out)
    ctx.sync()
    y = y.double().cpu().numpy()
    for r in range(R):
        if (y[r] == -np.inf).all():
            assert t[r] == -1
            continue
        p = np.exp((y[r] - y[r].max()) / temperature)
        cdf = np.cumsum(p) / p.sum()
        j = int(t[r])
        u = oracle.philox_uniform(11, r, 0, 1 << 33)
        assert p[j] > 0 and (cdf[j - 1] if j else 0) - 1e-5 <= u <= cdf[j] + 1e-5


def test_draws_follow_the_split_heads(sph, ctx):
    # the same logits through the endpoint's draw and through this one: the same uniforms,
    # so the same tokens but where a draw lies within rounding of a step
    R, d, n = 50, 64, 3000
    g = torch.Generator(device=DEV).manual_seed(1)
    h = torch.randn(R, d, generator=g, device=DEV)
    W = torch.randn(n, d, generator=g, device=DEV).to(torch.bfloat16)
    z = torch.empty(R, n, device=DEV)
    want = ctx.fuse_sample(None, None, h, W, temperature=0.9, seed=5, offset=2, fused_logits_out=z)
    y, got = ctx.shape_logits(z, n, temperature=0.9, seed=5, offset=2)
    ctx.sync()
    assert torch.equal(y, z) and int((want == got).sum()) >= R - 1


def test_long_histories_and_many_biases(ctx):
    R, n = 3, 5000
    z, a = make(R, n, n, 2, tokens=30000, biases=1000)
    y = call(ctx, dev(z, torch.float32), n, a)
    ctx.sync()
    assert same(y.cpu().numpy(), ora.shape(z, n, **a, dtype=np.float32))


@pytest.mark.parametrize("R,n", [(2, 40000), (310, 17000), (160, 70000)])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_marks_on_both_sides_of_a_block(ctx, R, n, off):
    # tokens around the borders of what a block counts, rows that begin off 16 bytes
    borders = [b for b in (16384, 32768, 65536) if b < n]
    near = np.array([b + k for b in borders for k in range(-9, 9)] + [0, n - 1])
    rng = np.random.default_rng(n)
    z = np.float32(rng.standard_normal((R, n)))
    h = near[rng.integers(0, len(near), (R, 30))]
    zd = torch.zeros(R, n + 4, device=DEV)
    zd[:, off:off + n] = dev(z, torch.float32)
    out = torch.empty(R, n + 4, device=DEV)[:, off:off + n]
    a = dict(history=h, frequency=np.full(R, 0.5, np.float32), presence=np.full(R, 8.0, np.float32))
    y, t = call(ctx, zd[:, off:off + n], n, a, out=out, temperature=0.0)
    ctx.sync()
    want = z.copy()
    for r in range(R):
        v, c = np.unique(h[r], return_counts=True)
        want[r, v] = want[r, v] - np.float32(0.5) * c.astype(np.float32) - np.float32(8)
    assert same(y.cpu().numpy(), want) and t.tolist() == want.argmax(1).tolist()


def test_strided_lists(ctx):
    R, n = 4, 600
    z, a = make(R, n, n, 2, tokens=21, biases=6)
    want = ora.shape(z, n, **a, dtype=np.float32)
    wide = lambda k, t: torch.cat([dev(a[k], t), torch.zeros(R, 3, dtype=t, device=DEV)], 1)
    h, bi, bv, m = (wide(k, t) for k, t in (("history", torch.int32), ("bias_ids", torch.int32),
                                            ("bias_values", torch.float32), ("mask", torch.int32)))
    y = ctx.shape_logits(dev(z, torch.float32), n, history=h[:, :21], lengths=dev(a["lengths"], torch.int32),
                         prompt_lengths=dev(a["prompts"], torch.int32),
                         repetition=dev(a["repetition"], torch.float32),
                         frequency=dev(a["frequency"], torch.float32),
                         presence=dev(a["presence"], torch.float32), bias_ids=bi[:, :6],
                         bias_values=bv[:, :6], mask=m[:, :-(-n // 32)])
    ctx.sync()
    assert same(y.cpu().numpy(), want)


def test_no_tokens_yet(ctx):
    z, a = make(3, 100, 100, 2, tokens=5, biases=0, mask=0)
    a["history"] = np.zeros((3, 0), np.int64)
    a["lengths"] = a["prompts"] = np.zeros(3, np.int64)
    y, t = call(ctx, dev(z, torch.float32), 100, a, temperature=0.0)
    ctx.sync()
    assert same(y.cpu().numpy(), z) and t.tolist() == z.argmax(1).tolist()


def test_far_rows(ctx):
    # more than 2^31 logits
    R, n = 5, 1 << 29
    z = torch.zeros(R, n, dtype=torch.bfloat16, device=DEV)
    z[R - 1, n - 1], z[R - 1, 0], z[2, 5] = 3.0, 2.0, 1.0
    h = torch.full((R, 2), n - 1, dtype=torch.int32, device=DEV)
    y, t = ctx.shape_logits(z, n, history=h, presence=torch.full((R,), 0.5, device=DEV), temperature=0.0,
                            dtype=torch.float32)
    ctx.sync()
    assert t.tolist() == [0, 0, 5, 0, n - 1] and float(y[R - 1, n - 1]) == 2.5
    assert float(y[2, n - 1]) == -0.5 and int((y[3] != 0).sum()) == 1


def test_streams_and_graphs(sph, ctx):
    z, a = make(6, 4000, 4000, 9)
    zd = dev(z, torch.float32)
    want = call(ctx, zd, 4000, a, temperature=0.8, seed=1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call(ctx, zd, 4000, a, temperature=0.8, seed=1)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    own = sph.Context(0)
    own.reserve(6, 4000, 8)
    hist, mask = dev(a["history"], torch.int32), dev(a["mask"], torch.int32)
    rep = dev(a["repetition"], torch.float32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = own.shape_logits(zd, 4000, history=hist, repetition=rep, mask=mask, temperature=0.8, seed=1)
    for k in range(2):
        zd.copy_(dev(make(6, 4000, 4000, 20 + k)[0], torch.float32))
        g.replay()
        torch.cuda.synchronize()
        want = ctx.shape_logits(zd, 4000, history=hist, repetition=rep, mask=mask, temperature=0.8, seed=1)
        assert all(torch.equal(p, q) for p, q in zip(want, got))
    own.close()


def test_refusals(sph, ctx):
    z = torch.zeros(3, 100, device=DEV)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    f = lambda *s: torch.zeros(*s, device=DEV)
    bad = [lambda: ctx.shape_logits(z, 99), lambda: ctx.shape_logits(z.double(), 100),
           lambda: ctx.shape_logits(z, 200, keep_ids=i(99)),
           lambda: ctx.shape_logits(z, 100, history=i(2, 5)), lambda: ctx.shape_logits(z, 100, history=f(3, 5)),
           lambda: ctx.shape_logits(z, 100, history=i(3, 5), lengths=i(2)),
           lambda: ctx.shape_logits(z, 100, history=i(3, 5), repetition=f(3).double()),
           lambda: ctx.shape_logits(z, 100, bias_ids=i(3, 2)),
           lambda: ctx.shape_logits(z, 100, bias_ids=i(3, 2), bias_values=f(3, 3)),
           lambda: ctx.shape_logits(z, 100, mask=i(3, 3)), lambda: ctx.shape_logits(z, 100, tokens=i(3)),
           lambda: ctx.shape_logits(z, 100, temperature=0.0, tokens=i(2)),
           lambda: ctx.shape_logits(z, 100, out=f(3, 99)),
           lambda: ctx.shape_logits(z, 100, history=i(3, 5).cpu())]
    for c in bad:
        with pytest.raises(ValueError):
            c()
    for c in (lambda: ctx.shape_logits(z, 100, repetition=f(3)), lambda: ctx.shape_logits(z, 100, mask=i(2, 4)),
              lambda: ctx.shape_logits(z, 100, mask_rows=i(3)), lambda: ctx.shape_logits(z[:0], 100),
              lambda: ctx.shape_logits(z, 100, temperature=-1.0),
              lambda: ctx.shape_logits(z, 100, temperature=float("nan")),
              lambda: ctx.shape_logits(z, 100, temperature=0.0, dtype=torch.bfloat16)):
        with pytest.raises(sph.SphError):
            c()
    c = sph.Context(0)
    c.set_option(sph.SPH_OPT_SAMPLER, 1)
    with pytest.raises(sph.SphError):
        c.shape_logits(z, 100, temperature=1.0)
    c.close()


def test_a_step_from_hidden_states_to_the_next_inputs(sph, ctx):
    # norm, product with a table in e4m3 blocks, penalties, mask and token, lookup: as a
    # decoding step runs them, against the same steps in 64 bits
    R, V, d = 7, 900, 384
    rng = np.random.default_rng(4)
    x = dev(rng.standard_normal((R, d)) * 3 + 1, torch.bfloat16)
    w = dev(1 + 0.2 * rng.standard_normal(d), torch.float32)
    table = ctx.fp8_quantize(dev(rng.standard_normal((V, d)) * 0.05, torch.float32), 128)
    _, a = make(R, V, V, 8, tokens=30, biases=4, mask=0.7)
    h = ctx.layer_norm(x, w, centre=False, dtype=torch.float32)
    z = ctx.fp8_logits(h, table)
    y, t = call(ctx, z, V, a, temperature=0.0)
    e = ctx.embed(t, table, scale=2.0, dtype=torch.float32)
    ctx.sync()
    h64 = h.double().cpu().numpy()
    assert np.abs(h64 - ora.norm(x.double().cpu().numpy(), w.double().cpu().numpy(), centre=False)[0]).max() < 1e-5
    t64 = ora.decode8(table.codes.view(torch.uint8).cpu().numpy(), table.scales.cpu().numpy(), 128)
    want, mag = ora.product8(h64, t64)
    assert (np.abs(z.double().cpu().numpy() - want) <= 300 * 2.0 ** -24 * mag).all()
    shaped = ora.shape(z.cpu().numpy(), V, **a, dtype=np.float32)
    assert same(y.cpu().numpy(), shaped) and t.tolist() == first_largest(shaped, None)
    assert np.abs(e.double().cpu().numpy() - 2 * t64[t.cpu().numpy()]).max() < 1e-6
