"""Host checks of the binding of the operators around the head's product: what the native
marshalling does not take goes to Python, which refuses it (no GPU needed)."""
import ctypes
import os
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
    x, v = torch.zeros(2, 32), torch.zeros(32)
    w = sph.fp8_empty(4, 32, device="cpu")
    for handle in (None, 0, 1, 1.5, object()):
        assert f.fp8_quantize(handle, x, 1) == no
        assert f.fp8_dequantize(handle, w, None, None) == no
        assert f.fp8_logits(handle, x, w, None, None, None, None) == no
        assert f.embed(handle, torch.zeros(2, dtype=torch.int32), w, 1.0, -1, None, None) == no
        assert f.layer_norm(handle, x, v, v, 1e-5, True, True, None, None) == no
        assert f.layer_norm_grad(handle, x, x, v, v[:2], v[:2], True, False, *[None] * 5) == no
        assert f.shape_logits(handle, x, 32, *[None] * 12, 0, 0, *[None] * 3) == no
    for call in (f.fp8_quantize, f.fp8_dequantize, f.fp8_logits, f.layer_norm, f.layer_norm_grad,
                 f.shape_logits):
        assert call() == no and call(1) == no
        for n in range(2, 23):
            for what in (object(), None, (), (1, 2, 3), 1, 1.5, True, x):
                assert call(*[what] * n) == no


def test_python_refuses_host_tensors(sph):
    x, v = torch.zeros(2, 32), torch.zeros(32)
    w = sph.fp8_empty(4, 32, device="cpu")
    for call in (lambda: sph.sph_fp8_quantize(None, x), lambda: sph.sph_fp8_dequantize(None, w),
                 lambda: sph.sph_fp8_logits(None, x, w), lambda: sph.sph_layer_norm(None, x, v),
                 lambda: sph.sph_embed(None, torch.zeros(2, dtype=torch.int32), w),
                 lambda: sph.sph_layer_norm_grad(None, x, x, v, v[:2], v[:2]),
                 lambda: sph.sph_shape_logits(None, x, 32)):
        with pytest.raises(ValueError):
            call()


def test_room_for_rows(sph):
    for rows, d, block, ld, scales in ((3, 1, 1, 16, (3, 1)), (129, 129, 128, 144, (2, 2)),
                                       (128, 128, 128, 128, (1, 1)), (2, 4097, 1, 4112, (2, 33))):
        w = sph.fp8_empty(rows, d, block, device="cpu")
        assert tuple(w.codes.shape) == (rows, d) and w.codes.stride(0) == ld
        assert tuple(w.scales.shape) == scales and w.block_rows == block
    for bad in ((0, 4, 1), (4, 0, 1), (4, 4, 2), (4, 4, 0)):
        with pytest.raises(ValueError):
            sph.fp8_empty(*bad, device="cpu")


def test_structs_follow_the_header(sph):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "sph.h")).read(), flags=re.S)
    kinds = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32}
    for name in ("sph_fp8", "sph_shaping"):
        body = re.search(r"typedef struct %s \{(.*?)\}" % name, text, flags=re.S).group(1)
        fields = re.findall(r"((?:const\s+)?\w+\s*\*?)\s*(\w+)\s*;", body)
        want = [(n, ctypes.c_void_p if "*" in t else kinds[t.strip()]) for t, n in fields]
        assert want == getattr(sph, name)._fields_


def test_null_context_is_refused(sph):
    assert sph.lib.sph_fp8_quantize(None, None, 0, 0, None) == 1
    assert sph.lib.sph_embed_fp8(None, None, 0, None, 1.0, -1, None, 0, 0) == 1
    assert sph.lib.sph_fp8_logits(None, None, 0, 0, 0, None, None, None, 0, None, 0, 0) == 1
    assert sph.lib.sph_layer_norm(None, None, 0, 0, 0, 0, None, None, 0, 0.0, 1, None, 0, 0, None,
                                  None) == 1
    assert sph.lib.sph_layer_norm_grad(None, None, 0, 0, None, 0, 0, 0, 0, None, 0, None, None, None,
                                       0, 0, None, None, 0, 0) == 1
    assert sph.lib.sph_shape_logits(None, None, 0, 0, 0, None, 0, 0, None, None, 0, 0, 0.0, 0, 0,
                                    None) == 1
