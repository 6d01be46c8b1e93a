"""Host side of the rotary and scored-attention calls: the frequencies that he_rotary_init makes, and every refusal that needs no GPU."""
import ctypes
import math

import pytest

from paper_2412_16187_b200 import HashEvictError, Rotary, binding

TURN = 1 << 64


def frequencies(r, base, kind=None, factor=1.0, length=8192.0, low=1.0, high=32.0):
    """The definitions in include/hashevict.h, in Python's 64 bits."""
    if kind == "ntk":
        base *= factor ** (r / (r - 2))
    f = [base ** (-2 * i / r) for i in range(r // 2)]
    if kind == "linear":
        return [x / factor for x in f], 1.0
    if kind == "yarn":
        at = lambda turns: r * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
        ramp = [min(max((i - a) / max(b - a, 0.001), 0.0), 1.0) for i in range(r // 2)]
        return [x / factor * t + x * (1 - t) for x, t in zip(f, ramp)], 0.1 * math.log(factor) + 1.0
    if kind == "bands":
        mix = [min(max((length * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        return [(1 - m) * x / factor + m * x for x, m in zip(f, mix)], 1.0
    return f, 1.0


@pytest.mark.parametrize("channels", [2, 10, 64, 96, 128, 256])
@pytest.mark.parametrize("scaling", [None, {"kind": "linear", "factor": 4.0}, {"kind": "ntk", "factor": 8.0},
                                     {"kind": "yarn", "factor": 8.0, "length": 4096}, {"kind": "bands", "factor": 8.0, "length": 8192}])
def test_frequencies_are_those_of_the_definition(channels, scaling):
    if scaling and scaling["kind"] == "ntk" and channels == 2:
        with pytest.raises(HashEvictError, match="NTK"):
            Rotary(256, channels, base=500000.0, scaling=scaling)
        return
    kw = dict(scaling or {})
    if kw.get("kind") == "bands":
        kw["high"] = 4.0
    want, amplitude = frequencies(channels, 500000.0, **kw)
    raw = Rotary(256, channels, base=500000.0, interleaved=True, scaling=scaling).raw
    assert raw.channels == channels and raw.interleaved == 1 and raw.amplitude == ctypes.c_float(amplitude).value
    for i, f in enumerate(want):
        # 64-bit arithmetic on both sides: a few roundings of 2^-53 each of a frequency of at most 1 radian, and the step of 2^-64 turns
        assert abs(raw.turns[i] / TURN - f / (2 * math.pi)) <= 16 * 2.0 ** -53 * f + 2.0 ** -64, i
    assert not any(raw.turns[channels // 2:])


def test_given_frequencies_are_reduced_to_a_turn():
    raw = Rotary(64, 8, frequencies=[0.0, 1.0, -1.0, 2 * math.pi * 3.25], amplitude=0.5).raw
    assert raw.amplitude == 0.5 and raw.turns[0] == 0
    assert abs(raw.turns[1] / TURN - 1 / (2 * math.pi)) < 1e-15
    assert (raw.turns[1] + raw.turns[2]) % TURN in (0, 1, TURN - 1)  # a turn the other way
    assert abs(raw.turns[3] / TURN - 0.25) < 1e-14


@pytest.mark.parametrize("kw, text", [
    (dict(channels=7), "even"), (dict(channels=0), "even"), (dict(channels=130), "head_dim"), (dict(base=1.0), "base"), (dict(base=float("nan")), "base"),
    (dict(scaling={"kind": "linear", "factor": 0.5}), "factor"), (dict(scaling={"kind": "linear"}), "scaling"), (dict(scaling={"factor": 2.0}), "kind"),
    (dict(scaling={"kind": "spiral", "factor": 2.0}), "kind"), (dict(scaling={"kind": "linear", "factor": 2.0, "length": 8}), "scaling"),
    (dict(scaling={"kind": "yarn", "factor": 2.0}), "length"), (dict(scaling={"kind": "bands", "factor": 2.0, "length": 8, "low": 4, "high": 4}), "low"),
    (dict(frequencies=[1.0]), "frequencies"), (dict(channels=2, frequencies=[float("inf")]), "finite"), (dict(amplitude=2.0), "amplitude"),
    (dict(channels=2, frequencies=[1.0], amplitude=float("nan")), "amplitude"),
])
def test_rotary_refuses(kw, text):
    with pytest.raises(HashEvictError, match=text):
        Rotary(128, **kw)


FAKE = 0x10000  # never followed: every check below comes before the launch


def test_calls_refuse_on_the_host():
    L, err = binding.lib(), lambda: binding.lib().he_last_error().decode()
    i64x3, i64x2 = ctypes.c_int64 * 3, ctypes.c_int64 * 2
    ok3, ok2 = i64x3(8 * 64 * 16, 64 * 16, 64), i64x2(8 * 64, 64)  # [2, up to 8 heads, 16, 64]
    cfg = ctypes.byref(binding.he_config(2, 2, 4, 64, 32, 64, 0, 0, 1, 0))
    rot = ctypes.byref(Rotary(64).raw)
    wide = ctypes.byref(Rotary(128).raw)

    def prompt(rotary=rot, q=FAKE, k=FAKE, qs=ok3, ks=ok3, n=16, qo=FAKE, ko=FAKE, qos=ok3, kos=ok3):
        return L.he_rotate_prompt(cfg, rotary, q, k, qs, ks, None, None, n, qo, ko, qos, kos, None)

    assert prompt(rotary=None) == 1 and "rotary is null" in err()
    assert prompt(rotary=wide) == 1 and "head_dim" in err()
    assert prompt(n=-1) == 1 and "max_prompt_len" in err()
    assert prompt(n=0) == 0
    assert prompt(qo=None) == 1 and "null" in err()
    assert prompt(k=FAKE + 2) == 1 and "aligned" in err()
    assert prompt(qs=None) == 1 and "strides" in err()
    assert prompt(ks=i64x3(64, 64, 4)) == 1 and "aligned" in err()
    assert prompt(ks=i64x3(64, -64, 64)) == 1 and "stride" in err()
    assert prompt(qos=i64x3(9 * 64 * 16, 64 * 16, 64)) == 1 and "in place" in err()
    for bad in (i64x3(64 * 16, 64, 0), i64x3(64 * 16, 64, 64), i64x3(64, 64 * 16, 64), i64x3(2 * 64 * 16 - 8, 64 * 16, 64)):
        assert prompt(kos=bad) == 1 and "overlap" in err()
    assert prompt(n=1, ks=i64x3(128, 64, 0), kos=i64x3(64, 64, 0)) == 1 and "overlap" in err()  # (of one token only its stride says nothing)

    cache = binding.he_cache()
    step = lambda c: L.he_rotate_step(cfg, rot, c, FAKE, FAKE, ok2, ok2, FAKE, FAKE, ok2, ok2, None)  # noqa: E731
    assert step(None) == 1 and "null" in err()
    assert step(ctypes.byref(cache)) == 1 and "next_pos" in err()

    def attend(mod=None, q=FAKE, v=FAKE, qs=ok3, kvs=ok3, lens=FAKE, n=16, out=FAKE, os=ok3, c=cfg):
        return L.he_attend_prompt(c, None if mod is None else ctypes.byref(mod), q, FAKE, v, qs, kvs, lens, n, None, None, out, os, None)

    mod = binding.he_score_mod
    assert attend(n=-1) == 1 and "max_prompt_len" in err()
    assert attend(n=(1 << 24) + 1) == 2 and "2^24" in err()
    assert attend(n=0, q=None) == 0
    assert attend(q=None) == 1 and attend(v=None) == 1 and attend(lens=None) == 1 and attend(out=None) == 1 and "null" in err()
    assert attend(v=FAKE + 8) == 1 and "aligned" in err()
    assert attend(kvs=i64x3(64, 64, 12)) == 1 and "aligned" in err()
    assert attend(os=None) == 1 and "out strides" in err()
    assert attend(os=i64x3(64 * 16, 0, 64)) == 1 and "overlap" in err()
    assert attend(os=i64x3(64 * 8, 64, 64)) == 1 and "overlap" in err()
    for bad, word in ((mod(-1.0, 0, 0, 0, None), "scale"), (mod(float("nan"), 0, 0, 0, None), "scale"), (mod(0, -2.0, 0, 0, None), "cap"),
                      (mod(0, float("inf"), 0, 0, None), "cap"), (mod(0, 0, -1, 0, None), "window"), (mod(3e38, 1e-30, 0, 0, None), "leaves fp32")):
        assert attend(mod=bad) == 1 and word in err(), word
        full = binding.he_cache(*([FAKE] * 9), None, None)
        assert L.he_attend_scored(cfg, ctypes.byref(full), ctypes.byref(bad), FAKE, None, FAKE, None) == 1 and word in err(), word
    assert L.he_attend_scored(cfg, ctypes.byref(cache), None, FAKE, None, FAKE, None) == 1 and "null" in err()
    full = binding.he_cache(*([FAKE] * 9), None, None)
    assert L.he_attend_scored(cfg, ctypes.byref(full), None, FAKE + 4, None, FAKE, None) == 1 and "aligned" in err()
    many = binding.he_config(70000, 2, 4, 64, 32, 64, 0, 0, 1, 0)
    assert L.he_attend_scored(ctypes.byref(many), ctypes.byref(full), None, FAKE, None, FAKE, None) == 2 and "65535" in err()
