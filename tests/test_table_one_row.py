"""Tables of one row in 4 bits: the binding refuses codes and scales whose bytes do not lie
one after the other, whatever the number of rows (no GPU needed)."""
import pytest
import torch


@pytest.fixture(scope="module")
def sph():
    from paper_2607_13093_gb300 import build_lib
    build_lib.build()
    from paper_2607_13093_gb300 import sph as m
    return m


class OnDevice:
    """A host tensor that says it lies on the GPU: enough for the argument checks."""
    device, is_cuda = torch.device("cuda", 0), True

    def __init__(self, t):
        self._t = t

    def __getattr__(self, name):
        return getattr(self._t, name)


def table(sph, codes, scales, rows):
    return sph.Mx4(OnDevice(codes), OnDevice(scales), OnDevice(torch.ones(rows)), 64, sph.SPH_MX4_E4M3)


def views(rows, n):
    """Views of [rows, n] bytes that are not dense rows, and one that is."""
    return [torch.zeros(rows, 2 * n, dtype=torch.uint8)[:, ::2],
            torch.zeros(rows, 1, dtype=torch.uint8).expand(rows, n),
            torch.zeros(n, rows + 1, dtype=torch.uint8).t()[:rows]], \
        torch.zeros(rows, n + 16, dtype=torch.uint8)[:, :n]


@pytest.mark.parametrize("rows", [1, 2])
def test_rows_that_are_not_dense_are_refused(sph, rows):
    (bad_codes, codes), (bad_scales, scales) = views(rows, 32), views(rows, 16)
    c = sph._mx4(table(sph, codes, scales, rows), OnDevice.device)
    assert (c.codes, c.scales, c.rows, c.d) == (codes.data_ptr(), scales.data_ptr(), rows, 64)
    assert c.ld_codes >= 32 and c.ld_scales >= 16 and c.ld_codes % 16 == c.ld_scales % 16 == 0
    for b in bad_codes:
        with pytest.raises(ValueError):
            sph._mx4(table(sph, b, scales, rows), OnDevice.device)
    for b in bad_scales:
        with pytest.raises(ValueError):
            sph._mx4(table(sph, codes, b, rows), OnDevice.device)
    with pytest.raises(ValueError):
        sph._mx4(table(sph, codes[0], scales, rows), OnDevice.device)
