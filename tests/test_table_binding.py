"""Host checks of the table operators' binding: what the native marshalling does not
take goes to Python, which refuses it (no GPU needed)."""
import re

import pytest
import torch


@pytest.fixture(scope="module")
def sph():
    from paper_2607_13093_gb300 import build_lib
    build_lib.build()
    from paper_2607_13093_gb300 import sph as m
    return m


def test_anything_not_plain_is_left_to_python(sph):
    f, no = sph._fast, sph._NOT_TAKEN
    x, tok = torch.zeros(2, 32), torch.zeros(2, dtype=torch.int32)
    w = sph.Mx4(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 16, dtype=torch.uint8),
                torch.ones(4), 32, sph.SPH_MX4_E4M3)
    for handle in (None, 0, 1, 1.5, object()):
        assert f.mx4_quantize(handle, x, sph.SPH_MX4_E4M3) == no
        assert f.mx4_dequantize(handle, w, None, None) == no
        assert f.mx4_logits(handle, x, w, None, None, 2, None, None) == no
        assert f.embed(handle, tok, x, 1.0, -1, None, None) == no
        assert f.embed(handle, tok, w, 1.0, -1, None, None) == no
        assert f.embed_grad(handle, tok, x, 4, 1.0, -1, False, None, None) == no
    for call in (f.mx4_quantize, f.mx4_dequantize, f.mx4_logits, f.embed, f.embed_grad):
        assert call() == no and call(1) == no
        for n in range(2, 12):
            assert call(*[object()] * n) == no and call(*[None] * n) == no
            assert call(*[()] * n) == no and call(*[(1, 2, 3, 4, 5)] * n) == no


def test_python_refuses_host_tensors(sph):
    x, tok = torch.zeros(2, 32), torch.zeros(2, dtype=torch.int32)
    w = sph.mx4_empty(4, 32, sph.SPH_MX4_E8M0, device="cpu")
    for call in (lambda: sph.sph_mx4_quantize(None, x), lambda: sph.sph_mx4_dequantize(None, w),
                 lambda: sph.sph_mx4_logits(None, x, w), lambda: sph.sph_embed(None, tok, x),
                 lambda: sph.sph_embed_grad(None, tok, x, 4)):
        with pytest.raises(ValueError):
            call()


def test_room_for_rows(sph):
    for fmt, d, codes, scales in ((sph.SPH_MX4_E4M3, 1, 16, 16), (sph.SPH_MX4_E4M3, 256, 128, 16),
                                  (sph.SPH_MX4_E4M3, 257, 144, 32), (sph.SPH_MX4_E8M0, 512, 256, 16),
                                  (sph.SPH_MX4_E8M0, 513, 272, 32)):
        w = sph.mx4_empty(3, d, fmt, device="cpu")
        assert tuple(w.codes.shape) == (3, codes) and tuple(w.scales.shape) == (3, scales)
        assert (w.row_scale is None) == (fmt == sph.SPH_MX4_E8M0)
        assert w.block == (32 if fmt == sph.SPH_MX4_E8M0 else 16)
    for bad in ((0, 4, 3), (4, 0, 3), (4, 4, 2), (4, 4, 5)):
        with pytest.raises(ValueError):
            sph.mx4_empty(*bad, device="cpu")


def test_struct_and_constants_follow_the_header(sph):
    import ctypes
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "sph.h")).read(), flags=re.S)
    body = re.search(r"typedef struct sph_mx4 \{(.*?)\}", text, flags=re.S).group(1)
    fields = re.findall(r"(\w+\s*\*?)\s*(\w+)\s*;", body)
    kinds = {"void*": ctypes.c_void_p, "float*": ctypes.c_void_p, "int64_t": ctypes.c_int64,
             "int32_t": ctypes.c_int32}
    assert [(n, kinds[t.replace(" ", "")]) for t, n in fields] == sph.sph_mx4._fields_
    header = {m.group(1): int(m.group(2))
              for m in re.finditer(r"\b(SPH_(?:TAB|MX4)_[A-Z0-9]+)\s*=\s*(\d+)", text)}
    assert header == {k: v for k, v in vars(sph).items() if k.startswith(("SPH_TAB_", "SPH_MX4_"))}
