"""Calls around the cache that the library and its binding turn down before anything is launched."""
import ctypes

import pytest

from paper_2412_16187_b200 import HE_FLAG_EARLY_INPUTS, HashEvictError, Rotary, ScoreMod, binding

FAKE, FAR = 0x10000, 0x40000000  # never followed: every check below comes before the launch


def config(flags=0, dtype=1):
    return binding.he_config(2, 2, 4, 64, 32, 64, 0, 0, dtype, flags)


def test_a_step_that_reads_its_rows_early_is_not_rotated_for():
    L, cache, two = binding.lib(), binding.he_cache(*([FAKE] * 9), None, None), ctypes.c_int64 * 2
    q, k = two(8 * 64, 64), two(2 * 64, 64)
    for flags in (HE_FLAG_EARLY_INPUTS, HE_FLAG_EARLY_INPUTS | 1):
        cfg = config(flags)
        assert L.he_rotate_step(ctypes.byref(cfg), Rotary(64).pointer, ctypes.byref(cache), FAKE, FAKE, q, k, FAR, FAR + FAKE, q, k, None) == 1
        assert b"EARLY_INPUTS" in L.he_last_error()


def test_a_cap_whose_ratio_to_the_scale_is_no_normal_number_is_refused():
    L, mod = binding.lib(), binding.he_score_mod
    cache, three = binding.he_cache(*([FAKE] * 9), None, None), ctypes.c_int64 * 3
    q, k = three(8 * 64 * 16, 64 * 16, 64), three(2 * 64 * 16, 64 * 16, 64)
    cfg = config()
    for bad in (mod(1e-30, 1e30, 0, 0, None), mod(1e-10, 1e35, 0, 0, None), mod(1e-38, 2.0, 0, 0, None)):
        assert L.he_attend_prompt(ctypes.byref(cfg), ctypes.byref(bad), FAKE, FAKE, FAKE, q, k, FAKE, 16, None, None, FAR, q, None) == 1
        assert b"leaves fp32" in L.he_last_error()
        assert L.he_attend_scored(ctypes.byref(cfg), ctypes.byref(cache), ctypes.byref(bad), FAKE, None, FAR, None) == 1
        assert b"leaves fp32" in L.he_last_error()


@pytest.mark.parametrize("kw, name", [(dict(window=2 ** 32 + 5), "window"), (dict(window=-(2 ** 32)), "window"), (dict(window=2 ** 31), "window"),
                                      (dict(window=2.5), "window"), (dict(softcap=1e-50), "softcap"), (dict(scale=1e-46), "scale"), (dict(scale=-1e-60), "scale")])
def test_numbers_that_the_library_has_no_type_for(kw, name):
    """None of them may turn into another number, or into none, on the way."""
    with pytest.raises(HashEvictError, match=name):
        ScoreMod(**kw)
    with pytest.raises(HashEvictError, match="channels"):
        Rotary(2 ** 33, 2 ** 32 + 64)


def test_numbers_at_the_ends_of_their_types_are_taken():
    raw = ScoreMod(window=2 ** 31 - 1, softcap=1e-40, scale=1e38).raw
    assert raw.window == 2 ** 31 - 1 and raw.cap > 0.0 and ScoreMod(window=16.0, scale=0, softcap=0).raw.window == 16


def test_outputs_that_are_other_arguments_are_refused():
    L, cache = binding.lib(), binding.he_cache(*([FAKE] * 9), None, None)
    cfg, rot, two, three = config(), Rotary(64), ctypes.c_int64 * 2, ctypes.c_int64 * 3
    q3, k3, q2, k2 = three(8 * 64 * 16, 64 * 16, 64), three(2 * 64 * 16, 64 * 16, 64), two(8 * 64, 64), two(2 * 64, 64)
    a, b, c, d = FAKE, FAR, 2 * FAR, 3 * FAR
    for q, k, qo, ko in ((a, b, c, c), (a, b, b, c), (a, b, c, a), (a, b, b, a)):
        assert L.he_rotate_prompt(ctypes.byref(cfg), rot.pointer, q, k, q3, k3, None, None, 16, qo, ko, q3, k3, None) == 1 and b"overlap" in L.he_last_error()
        assert L.he_rotate_step(ctypes.byref(cfg), rot.pointer, ctypes.byref(cache), q, k, q2, k2, qo, ko, q2, k2, None) == 1 and b"overlap" in L.he_last_error()
    for out in (a, b, c):
        assert L.he_attend_prompt(ctypes.byref(cfg), None, a, b, c, q3, k3, d, 16, None, None, out, q3, None) == 1 and b"out overlaps" in L.he_last_error()
