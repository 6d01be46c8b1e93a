"""A paged cache without pages, or whose sequences have no room for any: nothing is held, or what is held reads as zeros."""
import ctypes
import math

import pytest
import torch

from paper_2412_16187_b200 import PagedCache, binding
from test_gpu_layer_ops import BF16, F32


def test_calls_without_a_table_or_pages_are_taken():
    """Nothing is launched: the pointers are none."""
    L, cfg = binding.lib(), binding.he_config(2, 2, 4, 64, 32, 64, 0, 0, 1, 0)
    strides = (ctypes.c_int64 * 3)(2048, 1024, 64)
    for eight in (0, 1):
        none = binding.he_pages(None, None, None, None, None, 0x10000, 0, 16, 0, eight)
        c, p = ctypes.byref(cfg), ctypes.byref(none)
        assert L.he_page_append(c, p, None, 0x10000, 0x20000, strides, None, 3, None) == 0 and L.he_page_read(c, p, None, 3, 0x10000, 0x20000, strides, None) == 0
        assert L.he_page_attend_workspace_bytes(c, p) == 0
    for kw in (dict(max_pages=4), dict(n_pages=3), dict(len=None)):  # a table, or pages, that should be there
        f = {**dict(k_pages=0x10000, v_pages=0x10000, k_scale=0x10000, v_scale=0x10000, page_table=0x10000, len=0x10000, n_pages=0, page_size=16, max_pages=0, eight_bit=0), **kw}
        f["page_table" if "max_pages" in kw else "v_pages" if "n_pages" in kw else "len"] = None
        p = binding.he_pages(**f)
        assert L.he_page_append(c, ctypes.byref(p), None, 0x10000, 0x20000, strides, None, 3, None) == 1 and "null" in L.he_last_error().decode()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, eight, d", [(BF16, False, 64), (BF16, True, 128), (F32, False, 128), (F32, True, 64), (BF16, True, 256), (F32, False, 256)])
def test_nothing_is_held_or_zeros_are(dtype, eight, d):
    b, h, g, n = 3, 2, 3, 40
    q, k = torch.randn((b, h * g, d), device="cuda", dtype=dtype), torch.randn((b, h, n, d), device="cuda", dtype=dtype)
    for n_pages, per in ((0, 0), (0, 5), (8, 0)):
        cache = PagedCache(b, h, g, d, torch.zeros((b, per), dtype=torch.int32, device="cuda"), n_pages, 16, dtype=dtype, eight_bit=eight)
        cache.length += torch.tensor([n, 0, 17], dtype=torch.int32, device="cuda")
        cache.append(k, k)
        assert not cache.k_pages.view(torch.uint8).any() and not cache.v_pages.view(torch.uint8).any()
        out = torch.full((b, h * g, d), math.nan, device="cuda")
        assert not cache.attend(q, out=out).any()
        outs = [torch.full_like(k, 7.0) for _ in "kv"]
        cache.read(n, k_out=outs[0], v_out=outs[1])
        for x in outs:
            for s, held in enumerate((n, 0, 17)):
                some = held if per else 0
                assert not x[s, :, :some].any() and bool((x[s, :, some:] == 7.0).all())
