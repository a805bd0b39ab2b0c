"""The table's gradient of long token lists, whose sort takes several tiles a CTA.

Rows of d_out hold whole numbers from -4 to 4: at most 2^20 of them sum up below 2^24, so
every fp32 sum is exact in any order and the result has to be equal."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 8


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


def tokens(T, V, kind, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
    if kind == "falling":              # P(id) falls as 1 / (id + 1)
        t = ((V + 1.0) ** u - 1).long()
    elif kind == "uniform":
        t = (u * V).long()
    elif kind == "one id":
        t = torch.full((T,), V - 1, device=DEV)
    else:                              # in order, as one long text of its own vocabulary
        t = torch.arange(T, device=DEV) * V // T
    return t.clamp_(0, V - 1).to(torch.int32)


def rows(T, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-4, 5, (T, D), generator=g, device=DEV).float()


def want(t, d_out, V):
    keep = (t >= 0) & (t < V)
    y = torch.zeros(V, D, dtype=torch.float64, device=DEV)
    return y.index_add_(0, t[keep].long(), d_out[keep].double()).float()


# one digit's passes, two and three; each side of the 8 x 8192 tokens that the cluster holds
@pytest.mark.parametrize("V", [300, 70_000, 5_000_000])
@pytest.mark.parametrize("T", [65_535, 65_536, 65_537, 73_729, 200_000, 1 << 20])
@pytest.mark.parametrize("kind", ["falling", "uniform", "one id", "in order"])
def test_gradient_of_long_lists_is_exact(ctx, T, V, kind):
    t, d_out = tokens(T, V, kind, T), rows(T, V)
    t[::17] = -1
    got = ctx.embed_grad(t, d_out, V)
    assert torch.equal(got, want(t, d_out, V))
    for _ in range(4):
        assert torch.equal(ctx.embed_grad(t, d_out, V), got)


@pytest.mark.parametrize("T", [65_537, 1 << 20])
def test_long_lists_with_padding_inside_and_ids_outside(sph, ctx, T):
    V = 40_000
    t, d_out = tokens(T, V, "uniform", 1), rows(T, 2)
    t[5::7] = 123                                        # the padding id
    out = torch.full((V, D), 3.0, device=DEV)
    ctx.embed_grad(t, d_out, V, padding_id=123, accumulate=True, out=out)
    ctx.sync()
    keep = torch.where(t == 123, -1, t)
    assert torch.equal(out, want(keep, d_out, V) + 3)
    t[3::11], t[4::13] = V, -5                           # ids outside the table
    keep = torch.where(t == 123, -1, t)
    got = ctx.embed_grad(t, d_out, V, padding_id=123)
    with pytest.raises(sph.SphError) as e:
        ctx.sync()
    assert e.value.status == 1
    assert torch.equal(got, want(keep, d_out, V))
