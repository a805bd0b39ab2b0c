"""As many rows in 4 bits as the header admits, 2^31 - 1, of one column."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_the_largest_number_of_rows():
    import __graft_entry__ as g
    g.build()
    from paper_2607_13093_gb300 import sph
    rows = 2 ** 31 - 1                      # 34 GB of codes, as much of scales, 4 GB each way
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100e9:
        pytest.skip("needs 100 GB of device memory")
    ctx = sph.Context(0)
    # values that the form holds exactly: (4 or 6) times a power of two
    x = torch.tensor([1.0, -1.5, 0.0, 2.0, -3.0], dtype=torch.bfloat16, device=DEV)
    x = x.repeat(rows // 5 + 1)[:rows].view(rows, 1)
    w = ctx.mx4_quantize(x, sph.SPH_MX4_E8M0)
    back = ctx.mx4_dequantize(w)
    ctx.sync()
    assert torch.equal(back, x)
    del back
    assert bool((w.codes[-5:, 1:] == 0).all()) and bool((w.codes[-5:, 0] < 16).all())
    ctx.close()
    del x, w
    torch.cuda.empty_cache()
