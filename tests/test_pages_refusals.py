"""Calls of the paged cache and of attention over keys of another length that the library turns down before anything is launched."""
import ctypes

import pytest
import torch

from paper_2412_16187_b200 import Rotary, binding

FAKE, FAR = 0x10000, 0x40000000  # never followed: every call below is one that a check ends before the launch, and none is made where a launch could succeed
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="pointers that are none: without a GPU only")
three = ctypes.c_int64 * 3


def config(d=64, dtype=1, batch=2):
    return binding.he_config(batch, 2, 4, d, 32, 64, 0, 0, dtype, 0)


def pages(**kw):
    f = dict(k_pages=FAKE, v_pages=FAR, k_scale=FAKE, v_scale=FAKE, page_table=FAKE, len=FAKE, n_pages=8, page_size=16, max_pages=4, eight_bit=0)
    f.update(kw)
    return binding.he_pages(**f)


def calls(cfg, pg, k=FAKE, v=FAR, strides=three(2 * 64 * 16, 64 * 16, 64), n=16, rotary=None, out=FAR, q=FAKE, workspace=None, of=("append", "read", "attend")):
    """The error code and text of each of the calls that take pages."""
    L, found = binding.lib(), []
    c, p = (None if cfg is None else ctypes.byref(cfg)), (None if pg is None else ctypes.byref(pg))
    made = {"append": lambda: L.he_page_append(c, p, rotary, k, v, strides, None, n, None), "read": lambda: L.he_page_read(c, p, None, n, k, v, strides, None),
            "attend": lambda: L.he_page_attend(c, p, None, q, None, out, workspace, 0, None)}
    for name in of:
        found.append((made[name](), L.he_last_error().decode()))
    return found


@pytest.mark.parametrize("kw, code, text", [
    (dict(k_pages=None), 1, "null"), (dict(v_pages=None), 1, "null"), (dict(page_table=None), 1, "null"), (dict(len=None), 1, "null"), (dict(v_pages=FAR + 8), 1, "16-byte"),
    (dict(page_size=8), 1, "page_size"), (dict(page_size=48), 1, "page_size"), (dict(page_size=256), 1, "page_size"), (dict(page_size=-16), 1, "page_size"), (dict(n_pages=-1), 1, "n_pages"),
    (dict(max_pages=-1), 1, "max_pages"), (dict(max_pages=2 ** 20 + 1), 2, "2^24"), (dict(eight_bit=2), 1, "eight_bit"), (dict(eight_bit=1, k_scale=None), 1, "scales"),
    (dict(eight_bit=1, v_scale=None), 1, "scales")])
def test_pages(kw, code, text):
    for rc, said in calls(config(), pages(**kw)):
        assert rc == code and text in said


def test_shapes_and_pointers():
    for rc, said in calls(None, pages()):
        assert rc == 1 and "cfg" in said
    for rc, said in calls(config(), None):
        assert rc == 1 and "pages is null" in said
    for rc, said in calls(config(d=72), pages(eight_bit=1), strides=three(2 * 72 * 16, 72 * 16, 72)):
        assert rc == 2 and "multiple of 16" in said
    append, read = calls(config(), pages(), n=-1, of=("append", "read"))
    assert append[0] == read[0] == 1 and "max_new" in append[1] and "max_rows" in read[1]
    append, read, attend = calls(config(), pages(), k=None, v=None, q=None)
    assert append[0] == read[0] == attend[0] == 1 and "null" in append[1] and "neither" in read[1] and "null" in attend[1]
    append, read, attend = calls(config(), pages(), k=FAKE + 4, q=FAKE + 4)
    assert append[0] == read[0] == attend[0] == 1 and all("16-byte" in x[1] for x in (append, read, attend))
    for bad in (three(2 * 64 * 16, 64 * 16, 60), three(-64, 64, 64), None):
        append, read = calls(config(), pages(), strides=bad, of=("append", "read"))
        assert append[0] == read[0] == 1 and "stride" in append[1] and "stride" in read[1]
    assert "overlap" in calls(config(), pages(), strides=three(0, 64 * 16, 64), of=("read",))[0][1]
    assert "overlap" in calls(config(), pages(), v=FAKE, of=("read",))[0][1]
    assert calls(config(batch=70000), pages(), of=("read",))[0][0] == 2
    assert "out" in calls(config(), pages(), out=FAR + 8, of=("attend",))[0][1]
    assert "rotary channels 128" in calls(config(), pages(), rotary=Rotary(128).pointer, of=("append",))[0][1]


def test_calls_that_have_nothing_to_do_succeed_without_a_device():
    L, cfg = binding.lib(), config()
    c, p, none = ctypes.byref(cfg), ctypes.byref(pages()), ctypes.byref(pages(max_pages=0))
    assert L.he_page_append(c, p, None, None, None, None, None, 0, None) == 0 and L.he_page_append(c, none, None, FAKE, FAR, three(64, 64, 64), None, 3, None) == 0
    assert L.he_page_read(c, p, None, 0, None, None, None, None) == 0


def cross(cfg, mod=None, q=FAKE, k=FAR, v=2 * FAR, out=3 * FAR, qs=three(8 * 64 * 16, 64 * 16, 64), ks=three(2 * 64 * 32, 64 * 32, 64), q_len=FAKE, n=16, kv_len=FAKE, m=32, q_pos=None, first=None,
          prefix=None, os=None, workspace=None, size=0):
    L = binding.lib()
    rc = L.he_attend_cross(None if cfg is None else ctypes.byref(cfg), None if mod is None else ctypes.byref(mod), q, k, v, qs, ks, q_len, n, kv_len, m, q_pos, first, prefix, out,
                           qs if os is None else os, workspace, size, None)
    return rc, L.he_last_error().decode()


def test_rows_over_keys_of_another_length():
    cfg, mod = config(), binding.he_score_mod
    for bad in (mod(0, 0, 5, 0, None), mod(0, 0, 0, 0, FAKE)):
        assert cross(cfg, bad)[0] == 1 and "q_pos" in cross(cfg, bad)[1]
    assert cross(cfg, prefix=FAKE)[0] == 1 and "q_pos" in cross(cfg, prefix=FAKE)[1]
    assert cross(None) == (1, "cfg is null")
    for kw, code, text in ((dict(n=-1), 1, "max_q_len"), (dict(m=-1), 1, "max_kv_len"), (dict(n=2 ** 24 + 1), 2, "2^24"), (dict(m=2 ** 24 + 1), 2, "2^24"), (dict(q=None), 1, "null"), (dict(k=None), 1, "null"),
                           (dict(v=None), 1, "null"), (dict(out=None), 1, "null"), (dict(q_len=None), 1, "null"), (dict(kv_len=None), 1, "null"), (dict(q=FAKE + 8), 1, "16-byte"),
                           (dict(qs=three(64, 64, 60)), 1, "stride"), (dict(ks=None), 1, "stride"), (dict(os=three(64, 64, 0)), 1, "overlap"), (dict(out=FAR), 1, "overlaps"),
                           (dict(out=FAKE), 1, "overlaps"), (dict(workspace=FAKE + 8, size=64), 1, "workspace"), (dict(mod=mod(-1.0, 0, 0, 0, None)), 1, "scale")):
        rc, said = cross(cfg, **kw)
        assert rc == code and text in said, (kw, rc, said)
    assert cross(cfg, n=0)[0] == 0
    L = binding.lib()
    for n, m in ((0, 5), (5, 0), (-1, 5), (2 ** 24 + 1, 5)):
        assert L.he_attend_cross_workspace_bytes(ctypes.byref(cfg), n, m) == 0
