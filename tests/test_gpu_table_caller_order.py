"""The table operators read what they are given only after the caller's kernel
before them in the stream has written it, also where that kernel lets its
dependents start early and writes 50 us later (test_gpu_caller_order.py has the
writer), and calls that add to one gradient follow each other.  Needs a GPU
(marked gpu)."""
import pytest
import torch

from test_gpu_caller_order import ctx, writer  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu
DEV = "cuda"


def after(writer, dst, old, new, call):  # noqa: F811
    """call() with `new` in dst, written late while the caches hold `old`, and what it has to be."""
    dst.copy_(new)
    torch.cuda.synchronize()
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    for _ in range(3):
        dst.copy_(old)
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        writer(dst, new)
        got = call()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w)


def rand(*shape, dtype=torch.float32, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, device=DEV, generator=g).to(dtype)


def ids(n, V, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, V, (n,), device=DEV, generator=g, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [512, 514])
def test_quantise(ctx, writer, dtype, d):  # noqa: F811
    x = rand(300, d, dtype=dtype)
    after(writer, x, x.clone(), rand(300, d, dtype=dtype, seed=1), lambda: ctx.mx4_quantize(x)[:3])


@pytest.mark.parametrize("late", ["hidden", "codes", "scales", "row_scale", "ids"])
@pytest.mark.parametrize("rows", [3, 150])
@pytest.mark.parametrize("planes", [2, 4])
def test_logits(ctx, writer, late, rows, planes):  # noqa: F811
    V, d, n = 3000, 1024, 1000
    w, other = ctx.mx4_quantize(rand(V, d)), ctx.mx4_quantize(rand(V, d, seed=1) * 3)
    h = rand(rows, d, seed=2)
    keep = torch.arange(n, device=DEV, dtype=torch.int32) * 2
    dst, new = {"hidden": (h, rand(rows, d, seed=3)), "codes": (w.codes, other.codes),
                "scales": (w.scales, other.scales), "row_scale": (w.row_scale, other.row_scale),
                "ids": (keep, keep + 1000)}[late]
    after(writer, dst, dst.clone(), new,
          lambda: [ctx.mx4_logits(h, w, keep_ids=keep, planes=planes)])


@pytest.mark.parametrize("late", ["tokens", "table", "codes", "scales"])
@pytest.mark.parametrize("T", [20, 2000])
@pytest.mark.parametrize("d", [512, 514])
def test_lookup(ctx, writer, late, T, d):  # noqa: F811
    V = 700
    table, tok = rand(V, d, dtype=torch.bfloat16), ids(T, V)
    w, other = ctx.mx4_quantize(table), ctx.mx4_quantize(rand(V, d, seed=1) * 3)
    dst, new = {"tokens": (tok, ids(T, V, 1)), "table": (table, rand(V, d, dtype=torch.bfloat16, seed=1)),
                "codes": (w.codes, other.codes), "scales": (w.scales, other.scales)}[late]
    after(writer, dst, dst.clone(), new, lambda: [ctx.embed(tok, table), ctx.embed(tok, w)])


@pytest.mark.parametrize("late", ["tokens", "rows", "onto"])
@pytest.mark.parametrize("T", [100, 6000])
@pytest.mark.parametrize("d", [512, 514])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient(ctx, writer, late, T, d, dtype):  # noqa: F811
    V = 700
    tok, rows, onto = ids(T, V), rand(T, d, dtype=dtype), rand(V, d, dtype=dtype, seed=5)
    out = onto.clone()

    def call():
        if late == "onto":
            return [ctx.embed_grad(tok, rows, V, out=out, accumulate=True)]
        return [ctx.embed_grad(tok, rows, V, dtype=dtype)]

    dst, new = {"tokens": (tok, ids(T, V, 1)), "rows": (rows, rand(T, d, dtype=dtype, seed=1)),
                "onto": (out, rand(V, d, dtype=dtype, seed=6))}[late]
    after(writer, dst, dst.clone(), new, call)


@pytest.mark.parametrize("T", [100, 6000])
@pytest.mark.parametrize("d,wide", [(512, 512), (511, 511), (130, 133)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sums_added_many_times(ctx, T, d, wide, dtype):  # noqa: F811
    # ones: every sum is a whole number of sixteenths, which fp32 holds and bf16 rounds once a call
    V, calls = 700, 40
    tok = (torch.arange(T, device=DEV) % V).to(torch.int32)
    rows = torch.ones(T, d, device=DEV, dtype=dtype)
    out = torch.zeros(V, wide, device=DEV, dtype=dtype)[:, :d]
    for _ in range(calls):
        ctx.embed_grad(tok, rows, V, out=out, accumulate=True, scale=1.0 / 16)
    torch.cuda.synchronize()
    count = torch.bincount(tok.long(), minlength=V).float() * calls / 16
    exact = count[:, None].expand(V, d)
    if dtype == torch.bfloat16:
        assert ((out.float() - exact).abs() <= exact * calls * 2.0 ** -8).all()
    else:
        assert torch.equal(out, exact)
