"""Calls of the operators on 8-bit rows without the tensors that they need: refused as other wrong arguments are, without a GPU."""
import types

import pytest

torch = pytest.importorskip("torch")

import paper_2512_15550_amd as ck
from paper_2512_15550_amd import _marshal as M


def cache():
    shapes = {"pages": (3, 2, 16, 128), "cu": (2,), "batch": (1,), "table": (1, 3), "heads": (4,), "scales": (3, 2, 16)}

    def called(*_):
        raise AssertionError("the library was called")
    lib = types.SimpleNamespace(**{"ctkvr_cache_" + n: called for n in ("quant_append", "quant_read", "quant_attn", "window_attn", "tree_attn")})
    return types.SimpleNamespace(params=types.SimpleNamespace(n_q_heads=4, n_kv_heads=2, batch=1), torch_dtype=torch.bfloat16, _float=torch.float32, _int=torch.int32, device=-1,
                                 _pointer=M.pointer, _pointers=M.pointers, _rows=M.rows, _shapes=shapes, handle=1, n_axes=1, stream=lambda: 0, _lib=lib,
                                 _formats={torch.bfloat16: ck.KV_PLAIN, torch.int8: ck.KV_INT8, torch.float8_e4m3fn: ck.KV_FP8})


def arguments():
    codes, scales = torch.zeros((3, 2, 16, 128), dtype=torch.int8), torch.zeros((3, 2, 16))
    q, k = torch.zeros((5, 4, 128), dtype=torch.bfloat16), torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    batch = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 3), dtype=torch.int32)
    return codes, scales, q, k, batch


@pytest.mark.parametrize("k,v", [(False, False), (False, True)])
def test_rows_that_are_none(k, v):
    c, (codes, scales, q, kn, batch) = cache(), arguments()
    rows = [codes if k else None, scales if k else None, codes if v else None, scales if v else None]
    mask = torch.zeros((5, 1), dtype=torch.int32)
    for call in (lambda: ck.ctkvr_cache_quant_append(c, q, kn, kn, *batch, q, *rows), lambda: ck.ctkvr_cache_quant_attn(c, q, *rows, *batch, q),
                 lambda: ck.ctkvr_cache_window_attn(c, q, rows[0], rows[2], *batch, 7, q, k_scales=rows[1], v_scales=rows[3]),
                 lambda: ck.ctkvr_cache_tree_attn(c, q, rows[0], rows[2], *batch, mask, q, k_scales=rows[1], v_scales=rows[3])):
        with pytest.raises(ValueError, match="expected torch.int8"):
            call()


def test_nothing_to_append_or_to_read():
    c, (codes, scales, q, kn, batch) = cache(), arguments()
    pages = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k: expected"):
        ck.ctkvr_cache_quant_append(c, q, None, kn, *batch, q, codes, scales, codes, scales)
    with pytest.raises(ValueError, match="neither k_pages nor v_pages"):
        ck.ctkvr_cache_quant_read(c, codes, scales, codes, scales, batch[1], batch[2], batch[2], None, None)
    with pytest.raises(ValueError, match="expected torch.int8"):
        ck.ctkvr_cache_quant_read(c, None, None, None, None, batch[1], batch[2], batch[2], pages, pages)
