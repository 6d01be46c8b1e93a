"""Rotary positions, attention of prompts over themselves and scored attention over the cache against their definitions in 64 bits."""
import math

import pytest
import torch

from layer_reference import attend, prompt_seen, rotate, tolerance
from paper_2412_16187_b200 import HashEvictCache, HashEvictError, Rotary, ScoreMod
from paper_2412_16187_b200 import binding

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def make_cache(b, h, g, d, dtype, budgets=None, max_budget=None):
    return HashEvictCache(b, h, g, d, 16, [16] * b if budgets is None else budgets, torch.randn((d, 16)), dtype=dtype, max_budget=max_budget)


def rows(gen, b, heads, n, d, dtype, layout="heads", pad=0):
    """[b, heads, n, d]; "tokens": as a projection leaves them; `pad`: further channels between two rows of memory."""
    shape = (b, n, heads, d + pad) if layout == "tokens" else (b, heads, n, d + pad)
    x = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)[..., :d]
    return x.transpose(1, 2) if layout == "tokens" else x


def true_frequencies(rot):
    """What the struct holds, as radians per position (fp64)."""
    return torch.tensor([2 * math.pi * (t / 2 ** 64) for t in rot.raw.turns[: rot.channels // 2]], dtype=torch.float64, device="cuda"), rot.raw.amplitude


def check_rotated(got, x, pos, rot):
    freq, amp = true_frequencies(rot)
    want = rotate(x, pos, freq, amp, rot.interleaved)
    # The kernel's angle is within 2^-24 of a half turn (its rounding to fp32), the reference's within 2^-52 of up to 2^31 turns (3e-6 radians at the farthest
    # positions); sine, cosine, products and sums round in fp32: a few 1e-7 of the pair's length. Then one rounding to the output's type.
    a = x.double()[..., : rot.channels].abs().amax(-1, keepdim=True) * 2 * max(1.0, abs(amp))
    far = 2.0 ** -52 * pos.double().abs()[..., None] * 2 * math.pi
    tol = (1e-6 + far) * a + (2.0 ** -8 if x.dtype == BF16 else 2.0 ** -24) * want.abs()
    assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() - tol).max())
    assert torch.equal(got[..., rot.channels:], x[..., rot.channels:])  # what is not rotated is copied


ROTARIES = [(64, 64, False), (64, 16, True), (128, 128, False), (128, 32, True), (128, 64, False), (80, 20, False), (80, 80, True), (96, 24, False),
            (96, 36, True), (72, 10, False), (72, 72, True), (256, 256, False), (8, 2, False), (40, 6, True), (128, 126, False)]


@pytest.mark.parametrize("d, r, inter", ROTARIES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotate_prompt(d, r, inter, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d * 1000 + r)
    for b, h, g, n, layout, far in ((1, 1, 1, 1, "heads", 0), (3, 2, 3, 37, "tokens", 0), (2, 4, 1, 130, "heads", 2 ** 31 - 200)):
        cache, rot = make_cache(b, h, g, d, dtype), Rotary(d, r, base=500000.0, interleaved=inter, scaling={"kind": "yarn", "factor": 4.0, "length": 2048})
        pad = 8 if dtype == BF16 else 4
        q, k = rows(gen, b, h * g, n, d, dtype, layout, pad), rows(gen, b, h, n, d, dtype, layout)
        pos = torch.randint(-far, far + 1, (b, n), generator=gen, device="cuda").to(torch.int32) if far else None
        lens = torch.randint(0, n + 1, (b,), generator=gen, device="cuda").to(torch.int32)
        lens[-1] = n + 5  # longer than what is there: every row
        out = [torch.full_like(x, 7.0) for x in (q, k)]
        cache.rotate_prompt(rot, q, k, lens, positions=pos, q_out=out[0], k_out=out[1])
        at = pos if pos is not None else torch.arange(n, device="cuda").expand(b, n)
        for x, y in zip((q, k), out):
            for s in range(b):
                e = min(n, int(lens[s]))
                check_rotated(y[s, :, :e], x[s, :, :e], at[s, None, :e].expand(x.shape[1], -1), rot)
                assert bool((y[s, :, e:] == 7.0).all())  # rows behind the end are left
        # all rows, in place, only one of the two
        want, _ = cache.rotate_prompt(rot, q, None, positions=pos)
        mine = q.clone()
        got, none = cache.rotate_prompt(rot, mine, None, positions=pos, q_out=mine)
        assert none is None and got is mine and torch.equal(mine, want)
        _, only_k = cache.rotate_prompt(rot, None, k, positions=pos)
        check_rotated(only_k, k, at[:, None].expand(-1, h, -1), rot)


@pytest.mark.parametrize("d, r, inter", ROTARIES[:9])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotate_step(d, r, inter, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d + r)
    for b, h, g in ((1, 4, 1), (5, 2, 4), (33, 8, 7)):
        cache, rot = make_cache(b, h, g, d, dtype), Rotary(d, r, interleaved=inter)
        cache.next_pos.copy_(torch.randint(0, 2 ** 20, (b, h), generator=gen, device="cuda"))  # a position for each unit
        qkv = torch.randn((b, h * (g + 2), d), generator=gen, device="cuda", dtype=dtype)
        q, k = qkv[:, : h * g], qkv[:, h * g: h * (g + 1)]
        q2, k2 = cache.rotate_step(rot, q, k)
        check_rotated(q2, q, cache.next_pos.repeat_interleave(g, dim=1), rot)
        check_rotated(k2, k, cache.next_pos, rot)
        cache.rotate_step(rot, q, k, q_out=q, k_out=k)  # in place
        assert torch.equal(q, q2) and torch.equal(k, k2)


def test_a_rotation_keeps_what_attention_sees():
    """q . k after the rotation depends on the distance of the positions alone, at any offset."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache, rot = make_cache(1, 1, 1, 64, F32), Rotary(64, base=10000.0)
    q, k = rows(gen, 1, 1, 1, 64, F32), rows(gen, 1, 1, 1, 64, F32)
    at = lambda p, x: cache.rotate_prompt(rot, x, None, positions=torch.tensor([[p]], dtype=torch.int32, device="cuda"))[0].double()  # noqa: E731
    near = (at(17, q) * at(5, k)).sum()
    # both rows are off by at most 1e-6 of their length (see check_rotated)
    bound = 4e-6 * float(q.double().norm() * k.double().norm())
    for offset in (1000, 10 ** 6, 2 ** 31 - 100):
        assert abs(float((at(17 + offset, q) * at(5 + offset, k)).sum() - near)) <= bound


# ------------------------------------------------------------------------------------------------------------ prompts
OPTIONS = {
    "plain": {}, "cap": {"cap": 20.0}, "bias": {"slopes": True}, "window": {"window": 37}, "docs": {"docs": 50}, "prefix": {"prefix": 400},
    "cap + bias + docs": {"cap": 5.0, "slopes": True, "docs": 90}, "all": {"cap": 30.0, "slopes": True, "docs": 64, "prefix": 300, "window": 100, "scale": 0.3},
    "window + prefix": {"window": 1, "prefix": 1000},
}
# (B, H, G, d, dtype, lengths, layout): one token, block edges at 64, 128 and 256 and beside them, empty prompts, odd heads and sizes
SHAPES = [
    (1, 4, 1, 64, F32, [128], "heads"), (3, 1, 2, 40, F32, [1, 0, 65], "tokens"), (1, 1, 3, 256, BF16, [70], "heads"), (2, 2, 1, 200, F32, [63, 129], "heads"),
    (1, 1, 1, 128, BF16, [1], "heads"), (4, 2, 4, 128, BF16, [127, 128, 129, 257], "heads"), (3, 2, 3, 128, BF16, [300, 0, 511], "tokens"),
    (2, 1, 8, 64, BF16, [513, 640], "tokens"), (2, 2, 7, 80, BF16, [200, 385], "heads"), (1, 1, 1, 96, BF16, [1000], "tokens"), (2, 2, 2, 8, BF16, [5, 300], "heads"),
    (1, 2, 1, 120, BF16, [769], "heads"),
]


def prompt_case(shape, opt, seed=0, junk=True):
    b, h, g, d, dtype, lens, layout = shape
    gen = torch.Generator(device="cuda").manual_seed(seed + d)
    n = max(lens) + 3
    q, k, v = rows(gen, b, h * g, n, d, dtype, layout), rows(gen, b, h, n, d, dtype, layout), rows(gen, b, h, n, d, dtype, layout)
    k = k.mul_(2.0)
    kw = {"doc_start": None, "prefix_len": None}
    if "docs" in opt:
        cut = torch.rand((b, n), generator=gen, device="cuda") < 1 / opt["docs"]
        kw["doc_start"] = torch.where(cut, torch.arange(n, device="cuda"), 0).cummax(1).values.to(torch.int32)
        kw["doc_start"][:, 2:n:97] = 2 ** 30  # tokens of no document see nothing
        kw["doc_start"][:, 5:n:101] = -3
    if "prefix" in opt:
        kw["prefix_len"] = torch.tensor([m * opt["prefix"] // 1000 for m in lens], dtype=torch.int32, device="cuda")
        kw["prefix_len"][-1] += 2 ** 30 if opt["prefix"] == 1000 else 0  # longer than the prompt
    slopes = torch.exp2(-torch.arange(1, h * g + 1, device="cuda") * 8.0 / (h * g)) if opt.get("slopes") else None
    mod = ScoreMod(scale=opt.get("scale", 0.0), softcap=opt.get("cap", 0.0), window=opt.get("window", 0), slopes=slopes)
    plen = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if junk:  # what lies behind a prompt may be anything
        for s, m in enumerate(lens):
            for x, bad in ((q, math.nan), (k, math.inf), (v, math.nan)):
                x[s, :, m:] = bad
    return q, k, v, plen, mod, kw, slopes


def check_prompt(out, q, k, v, lens, opt, kw, slopes, g, split=False):
    for s, n in enumerate(lens):
        if n == 0:
            continue
        seen = prompt_seen(n, opt.get("window", 0), None if kw["doc_start"] is None else kw["doc_start"][s], 0 if kw["prefix_len"] is None else int(kw["prefix_len"][s]))
        at = torch.arange(n, device="cuda")
        for u in range(k.shape[1]):
            sl = slice(u * g, u * g + g)
            ref = attend(q[s, sl, :n], k[s, u, :n], v[s, u, :n], at, at, seen, opt.get("scale", 0.0), opt.get("cap", 0.0), None if slopes is None else slopes[sl])
            got = out[s, sl, :n].double()
            off = (got - ref).abs() - tolerance(ref, v[s, u, :n].double().abs().max(), out.dtype, split)
            assert bool((off <= 0).all()), (s, u, float(off.max()))
            assert not got[:, ~seen.any(1)].any()  # a row that sees nothing gives zeros


@pytest.mark.parametrize("opt", list(OPTIONS))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}x{s[3]}-{'bf16' if s[4] == BF16 else 'fp32'}-{max(s[5])}-{s[6]}")
@pytest.mark.parametrize("path", ["default", "generic"])
def test_attend_prompt(shape, opt, path, monkeypatch):
    b, h, g, d, dtype, lens, _ = shape
    tensor_cores = dtype == BF16 and d <= 128
    if path == "generic":
        if not tensor_cores:
            pytest.skip("the default path is already the generic kernel")
        monkeypatch.setenv("HE_DISABLE_ATTEND_MMA", "1")
    o = OPTIONS[opt]
    q, k, v, plen, mod, kw, slopes = prompt_case(shape, o)
    out = torch.full_like(q, 7.0)
    cache = make_cache(b, h, g, d, dtype)
    assert cache.attend_prompt(q, k, v, plen, mod=mod, out=out, **kw) is out
    check_prompt(out, q, k, v, lens, o, kw, slopes, g, split=path == "generic" or not tensor_cores)
    for s, n in enumerate(lens):
        assert bool((out[s, :, n:] == 7.0).all())


@pytest.mark.parametrize("shape", [(1, 1, 2, 128, BF16, [700], "heads"), (1, 2, 1, 64, BF16, [400], "tokens"), (1, 1, 2, 64, F32, [200], "heads")])
@pytest.mark.parametrize("opt", ["plain", "docs", "cap + bias + docs", "window", "prefix"])
def test_hidden_infinities_and_nans_touch_nobody(shape, opt):
    b, h, g, d, dtype, lens, _ = shape
    o = OPTIONS[opt]
    q, k, v, plen, mod, kw, slopes = prompt_case(shape, o, seed=5)
    n = lens[0]
    v[0, 0, n - 60, 3] = math.inf
    v[0, 0, n - 60, 5] = math.nan
    v[0, 0, n // 2, 7] = -math.inf
    cache = make_cache(b, h, g, d, dtype)
    out = cache.attend_prompt(q, k, v, plen, mod=mod, **kw)
    at = torch.arange(n, device="cuda")
    seen = prompt_seen(n, o.get("window", 0), None if kw["doc_start"] is None else kw["doc_start"][0], 0 if kw["prefix_len"] is None else int(kw["prefix_len"][0]))
    clean = v[:, :, :n].masked_fill(~torch.isfinite(v[:, :, :n]), 0.0)
    touched = seen[:, n - 60] | seen[:, n // 2]
    assert bool((~touched).any()) and bool(torch.isfinite(out[0, :g][:, :n][:, ~touched]).all())
    ref = attend(q[0, :g, :n], k[0, 0, :n], clean[0, 0], at, at, seen, o.get("scale", 0.0), o.get("cap", 0.0), None if slopes is None else slopes[:g])
    tol = tolerance(ref, clean[0, 0].abs().max().double(), dtype, dtype == F32)
    assert bool(((out[0, :g, :n].double() - ref).abs() <= tol)[:, ~touched].all())
    # those that see them have them, where the definition has them
    assert bool(torch.isnan(out[0, :g, :n, 5][:, seen[:, n - 60]]).all())


def test_attend_prompt_of_broadcast_and_strided_inputs():
    """KV heads that are one tensor seen several times (a stride of zero), and rows with gaps between them."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    b, h, g, d, n = 2, 3, 2, 128, 200
    cache = make_cache(b, h, g, d, BF16)
    q = rows(gen, b, h * g, n, d, BF16, "tokens", 64)
    one = rows(gen, b, 2, n, d, BF16, "heads", 16)
    k, v = one[:, :1].expand(-1, h, -1, -1), one[:, 1:].expand(-1, h, -1, -1)
    plen = torch.tensor([n, 131], dtype=torch.int32, device="cuda")
    out = cache.attend_prompt(q, k, v, plen)
    check_prompt(out, q, k, v, [n, 131], {}, {"doc_start": None, "prefix_len": None}, None, g)


@pytest.mark.parametrize("opt", ["plain", "all", "prefix"])
@pytest.mark.parametrize("shape", [(3, 4, 8, 128, BF16, [1100, 700, 3], "tokens"), (2, 20, 1, 64, BF16, [1500, 900], "heads"), (1, 2, 4, 128, BF16, [2700], "heads")])
def test_more_tiles_than_the_gpu_holds_at_once(shape, opt):
    """CTAs that go on from item to item: rings, phases and places carry over."""
    o = OPTIONS[opt]
    q, k, v, plen, mod, kw, slopes = prompt_case(shape, o, seed=3)
    out = torch.full_like(q, 7.0)
    make_cache(*shape[:5]).attend_prompt(q, k, v, plen, mod=mod, out=out, **kw)
    check_prompt(out, q, k, v, shape[5], o, kw, slopes, shape[2])
    for s, n in enumerate(shape[5]):
        assert bool((out[s, :, n:] == 7.0).all())


def test_prompts_without_tokens_and_rows_that_see_nothing():
    cache = make_cache(2, 1, 2, 128, BF16)
    q, k = torch.randn((2, 2, 300, 128), device="cuda").to(BF16), torch.randn((2, 1, 300, 128), device="cuda").to(BF16)
    out = torch.full_like(q, 7.0)
    for lens in ([0, 0], [-5, 0]):
        cache.attend_prompt(q, k, k, torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out)
        assert bool((out == 7.0).all())
    nothing = torch.full((2, 300), 10 ** 9, dtype=torch.int32, device="cuda")
    cache.attend_prompt(q, k, k, torch.tensor([300, 1000], dtype=torch.int32, device="cuda"), doc_start=nothing, out=out)
    assert not out.any()
    empty = cache.attend_prompt(q[:, :, :0], k[:, :, :0], k[:, :, :0], torch.tensor([3, 3], dtype=torch.int32, device="cuda"))
    assert empty.shape == (2, 2, 0, 128)


@pytest.mark.parametrize("cap, scale", [(0.25, 0.0), (1e6, 0.0), (3.0, 4.0), (50.0, 1e-7), (1e-3, 1.0), (2.0, 50.0)])
@pytest.mark.parametrize("dtype, d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_caps_far_from_the_scores(cap, scale, dtype, d):
    """Scores far inside the cap, about it and far beyond it, where tanh takes its other forms."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    n = 200
    cache = make_cache(1, 1, 2, d, dtype)
    q, k, v = rows(gen, 1, 2, n, d, dtype), rows(gen, 1, 1, n, d, dtype), rows(gen, 1, 1, n, d, dtype)
    out = cache.attend_prompt(q, k, v, torch.tensor([n], dtype=torch.int32, device="cuda"), mod=ScoreMod(scale=scale, softcap=cap))
    at = torch.arange(n, device="cuda")
    ref = attend(q[0], k[0, 0], v[0, 0], at, at, prompt_seen(n), scale=scale, cap=cap)
    # On the tensor cores tanh is within 7e-6 of itself (and 2e-6 absolutely): a score of x is off by at most 7e-6 |x|, with |x| <= min(cap, |raw|), and
    # fp32 products leave 1e-6 of the raw score. A weight is off by twice that, relatively, an output by as much of the largest |V|.
    raw = float((q[0].double() @ k[0, 0].double().T).abs().max()) * (scale or d ** -0.5)
    more = 2 * (7e-6 + 1e-6) * min(cap, raw) * float(v.double().abs().max())
    assert bool(((out[0].double() - ref).abs() <= tolerance(ref, v.double().abs().max(), dtype, dtype == F32) + more).all())


@pytest.mark.parametrize("dtype, d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_a_key_that_is_not_a_number_reaches_those_who_see_it(dtype, d):
    gen = torch.Generator(device="cuda").manual_seed(6)
    n, bad = 300, 140
    for mod, prefix in ((None, None), (ScoreMod(softcap=5.0), None), (ScoreMod(window=40), None), (ScoreMod(slopes=torch.ones(2, device="cuda")), 150)):
        cache = make_cache(1, 1, 2, d, dtype)
        q, k, v = rows(gen, 1, 2, n, d, dtype), rows(gen, 1, 1, n, d, dtype), rows(gen, 1, 1, n, d, dtype)
        k[0, 0, bad, 7] = math.nan
        pl = None if prefix is None else torch.tensor([prefix], dtype=torch.int32, device="cuda")
        out = cache.attend_prompt(q, k, v, torch.tensor([n], dtype=torch.int32, device="cuda"), mod=mod, prefix_len=pl)
        sees = prompt_seen(n, 40 if mod is not None and mod.raw.window else 0, None, prefix or 0)[:, bad]
        assert torch.equal(torch.isnan(out[0]).all(-1), sees.expand(2, -1)) and torch.equal(torch.isnan(out[0]).any(-1), sees.expand(2, -1))


# ---------------------------------------------------------------------------------------------- one token over the cache
def fill_cache(gen, shape, fills, junk=True):
    b, h, g, d, dtype = shape
    cache = make_cache(b, h, g, d, dtype, budgets=[max(f, 1) for f in fills], max_budget=max(max(fills), 4))
    cache.k_cache.copy_(torch.randn(cache.k_cache.shape, generator=gen, device="cuda") * 2)
    cache.v_cache.copy_(torch.randn(cache.v_cache.shape, generator=gen, device="cuda"))
    for s, f in enumerate(fills):
        for u in range(h):
            seen = 2 * f + u
            cache.fill[s, u], cache.next_pos[s, u] = f, seen
            if f:
                order = torch.randperm(seen, generator=gen, device="cuda")
                order = torch.cat((order[order == seen - 1], order[order != seen - 1]))[:f]
                cache.pos[s, u, :f] = order[torch.randperm(f, generator=gen, device="cuda")].to(torch.int32)
            if junk:
                cache.k_cache[s, u, f:], cache.v_cache[s, u, f:] = math.nan, math.inf
    return cache


def check_scored(got, cache, q, opt, slopes, first):
    g, h = cache.G, cache.H
    for s in range(cache.B):
        for u in range(h):
            f, now = int(cache.fill[s, u]), int(cache.next_pos[s, u]) - 1
            sl = slice(u * g, u * g + g)
            if f == 0:
                assert not got[s, sl].any()
                continue
            p = cache.pos[s, u, :f].long()
            seen = (p > now - opt["window"]) if opt.get("window") else torch.ones_like(p, dtype=torch.bool)
            if first is not None:
                seen = seen & (p >= first[s])
            v = cache.v_cache[s, u, :f]
            ref = attend(q[s, sl][:, None], cache.k_cache[s, u, :f], v, torch.tensor([now], device="cuda"), p, seen[None], opt.get("scale", 0.0), opt.get("cap", 0.0),
                         None if slopes is None else slopes[sl])[:, 0]
            if not seen.any():
                assert not got[s, sl].any()
                continue
            tol = tolerance(ref, v[seen].double().abs().max(), F32, True)
            assert bool(((got[s, sl].double() - ref).abs() <= tol).all()), (s, u, float((got[s, sl].double() - ref).abs().max()))


SCORED = {"plain": {}, "cap": {"cap": 20.0}, "bias": {"slopes": True}, "window": {"window": 33}, "first": {"first": 600}, "window of one": {"window": 1},
          "all": {"cap": 8.0, "slopes": True, "window": 200, "first": 300, "scale": 0.25}, "nothing seen": {"first": 5000}}


@pytest.mark.parametrize("opt", list(SCORED))
@pytest.mark.parametrize("shape, fills", [
    ((1, 4, 1, 64, F32), [64]), ((3, 2, 7, 256, BF16), [5, 0, 90]), ((2, 2, 3, 40, F32), [1, 130]), ((3, 2, 4, 128, BF16), [1, 33, 500]),
    ((1, 8, 4, 128, BF16), [2900]), ((2, 1, 8, 64, BF16), [700, 64]), ((2, 2, 5, 96, BF16), [333, 32]), ((200, 1, 2, 64, BF16), list(range(200))),
    ((2, 2, 2, 24, BF16), [100, 31]), ((2, 1, 1, 80, BF16), [1300, 1])], ids=lambda x: "x".join(map(str, x[:4])) if isinstance(x, tuple) else str(max(x)))
def test_attend_scored(shape, fills, opt):
    b, h, g, d, dtype = shape
    gen = torch.Generator(device="cuda").manual_seed(d + b)
    o = SCORED[opt]
    cache = fill_cache(gen, shape, fills)
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    slopes = torch.exp2(-torch.arange(1, h * g + 1, device="cuda") * 8.0 / (h * g)) if o.get("slopes") else None
    first = torch.tensor([2 * f * o["first"] // 1000 for f in fills], dtype=torch.int32, device="cuda") if "first" in o else None
    got = cache.attend_scored(q, ScoreMod(scale=o.get("scale", 0.0), softcap=o.get("cap", 0.0), window=o.get("window", 0), slopes=slopes), first_pos=first)
    check_scored(got, cache, q, o, slopes, first)
    if not o:  # he_attend's own result, in another kernel: both within 2e-5 of the largest |V| of exact arithmetic
        vmax = float(cache.v_cache[cache.pos >= 0].float().abs().max())
        assert torch.allclose(got, cache.attend(q), rtol=0, atol=4e-5 * vmax)


@pytest.mark.parametrize("opt", list(SCORED))
@pytest.mark.parametrize("shape, fills", [((3, 2, 4, 128, BF16), [1, 33, 500]), ((2, 3, 8, 64, BF16), [700, 64]), ((1, 1, 1, 104, BF16), [4100]), ((1, 2, 3, 256, F32), [1500])],
                         ids=lambda x: "x".join(map(str, x[:4])) if isinstance(x, tuple) else str(max(x)))
def test_attend_scored_without_tensor_maps(shape, fills, opt, monkeypatch):
    """The kernel of other types and head sizes, on shapes that the tensor-map kernel takes by default too; few units share CTAs."""
    monkeypatch.setenv("HE_DISABLE_ATTEND_MMA", "1")
    test_attend_scored(shape, fills, opt)


@pytest.mark.parametrize("shape", [(1, 2, 4, 128, BF16), (1, 1, 2, 64, F32), (1, 1, 2, 96, BF16)])
def test_hidden_slots_may_hold_anything(shape):
    b, h, g, d, dtype = shape
    gen = torch.Generator(device="cuda").manual_seed(9)
    cache = fill_cache(gen, shape, [300])
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    now = cache.next_pos[:, :, None] - 1
    hidden = (cache.pos >= 0) & (cache.pos <= now - 200)
    assert bool(hidden.any())
    want = cache.attend_scored(q, ScoreMod(window=200))
    cache.k_cache[hidden], cache.v_cache[hidden] = math.nan, -math.inf
    assert torch.equal(cache.attend_scored(q, ScoreMod(window=200)), want)


# ------------------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype, d", [(BF16, 128), (F32, 64)])
def test_a_layer_from_prompt_to_tokens(dtype, d):
    """Rotate, attend over the prompt and compress it, then token by token: rotate at the cache's position, evict, attend. With a budget that
    holds everything, the tokens' outputs are those of one long prompt; captured into a graph, everything is the same bit for bit."""
    b, h, g, n, more = 2, 2, 4, 190, 6
    gen = torch.Generator(device="cuda").manual_seed(11)
    w, lens = torch.randn((d, 16), generator=gen, device="cuda"), torch.tensor([n, n - 41], dtype=torch.int32, device="cuda")
    rot = Rotary(d, d // 2, base=10000.0, scaling={"kind": "linear", "factor": 2.0})
    slopes = torch.exp2(-torch.arange(1, h * g + 1, device="cuda").float())
    mod = ScoreMod(softcap=15.0, window=150, slopes=slopes)
    q, k, v = (rows(gen, b, x, n + more, d, dtype) for x in (h * g, h, h))
    # the long prompt of each sequence: its own tokens, then the new ones
    full = [torch.zeros_like(x) for x in (q, k, v)]
    for s in range(b):
        m = int(lens[s])
        for x, y in zip(full, (q, k, v)):
            x[s, :, :m], x[s, :, m:m + more] = y[s, :, :m], y[s, :, n:]

    def run(use_graph):
        cache = HashEvictCache(b, h, g, d, 16, [n + more] * b, w, dtype=dtype)
        st = torch.cuda.Stream()
        out_p = torch.zeros_like(q[:, :, :n])
        qp, kp = torch.zeros_like(q[:, :, :n]).contiguous(), torch.zeros_like(k[:, :, :n]).contiguous()
        outs = torch.zeros((more, b, h * g, d), device="cuda")
        vp, ws = v[:, :, :n].contiguous(), cache.workspace(n)
        steps = [[x[:, :, n + t].contiguous() for x in (q, k, v)] for t in range(more)]
        qt, kt, vic = torch.empty_like(steps[0][0]), torch.empty_like(steps[0][1]), torch.empty((b, h), dtype=torch.int32, device="cuda")

        def body():
            cache.rotate_prompt(rot, q[:, :, :n], k[:, :, :n], lens, q_out=qp, k_out=kp, stream=st)
            cache.attend_prompt(qp, kp, vp, lens, mod=mod, out=out_p, stream=st)
            cache.prefill_compress(qp, kp, vp, lens, n, workspace=ws, stream=st)
            for t in range(more):
                cache.rotate_step(rot, steps[t][0], steps[t][1], q_out=qt, k_out=kt, stream=st)
                cache.decode_step(qt, kt, steps[t][2], victim_out=vic, stream=st)
                cache.attend_scored(qt, mod, out=outs[t], stream=st)

        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            body()
            if use_graph:
                st.synchronize()
                out_p.zero_(), outs.zero_()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=st):
                    body()
                graph.replay()
                graph.replay()
        st.synchronize()
        return out_p, outs, cache.k_cache, cache.pos

    plain, graph = run(False), run(True)
    for x, y in zip(plain, graph):
        assert torch.equal(x, y)
    cache = make_cache(b, h, g, d, dtype)
    rq, rk = cache.rotate_prompt(rot, full[0], full[1])
    want = cache.attend_prompt(rq, rk, full[2], lens + more, mod=mod)
    vmax = float(v.abs().max())
    for s in range(b):
        m = int(lens[s])
        assert torch.equal(want[s, :, :m], plain[0][s, :, :m])
        for t in range(more):
            ref = want[s, :, m + t].double()
            # one is within tolerance() of exact arithmetic in the prompt's kernel, the other in the cache's; q and k are the same bits
            assert bool(((plain[1][t, s].double() - ref).abs() <= tolerance(ref, vmax, dtype, dtype == F32) + 2e-5 * vmax).all()), (s, t)


def test_two_streams_and_repeated_calls_give_the_same_bits():
    shape = (2, 2, 4, 128, BF16, [400, 650], "heads")
    o = OPTIONS["all"]
    q, k, v, plen, mod, kw, _ = prompt_case(shape, o, seed=2)
    cache = make_cache(2, 2, 4, 128, BF16)
    first = cache.attend_prompt(q, k, v, plen, mod=mod, out=torch.zeros_like(q), **kw)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(q) for _ in range(8)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        cache.attend_prompt(q, k, v, plen, mod=mod, out=out, stream=streams[i % 2], **kw)
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out, first)


@pytest.mark.parametrize("b, h, g, d, dtype", [(50, 8, 4, 128, BF16), (90, 4, 8, 64, BF16), (256, 2, 2, 96, BF16), (60, 8, 1, 64, F32), (300, 1, 4, 128, BF16)])
def test_the_order_of_the_units_changes_nothing(b, h, g, d, dtype):
    """With a mirror of the budgets the longest units start first; more units than the GPU holds at once, and more sequences than an order has room for."""
    gen = torch.Generator(device="cuda").manual_seed(b)
    budgets = torch.randint(1, 200, (b,), generator=torch.Generator().manual_seed(b))
    caches = [HashEvictCache(b, h, g, d, 16, budgets, torch.zeros((d, 16)), dtype=dtype, host_budget_mirror=m) for m in (False, True)]
    first, now = torch.randint(0, 150, (b,), generator=gen, device="cuda", dtype=torch.int32), 400
    k, v = (torch.randn(caches[0].k_cache.shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    pos = torch.randint(0, now, caches[0].pos.shape, generator=gen, device="cuda", dtype=torch.int32)
    q, mod = torch.randn((b, h * g, d), generator=gen, device="cuda").to(dtype), ScoreMod(softcap=10.0, window=350)
    outs = []
    for c in caches:
        c.k_cache.copy_(k), c.v_cache.copy_(v), c.pos.copy_(pos), c.next_pos.fill_(now)
        c.fill.copy_(budgets.to("cuda", torch.int32)[:, None].expand(b, h))
        outs.append(c.attend_scored(q, mod, first_pos=first))
    assert torch.equal(outs[0], outs[1])
    for s in (0, b // 2, b - 1):  # and against the definition
        n = int(budgets[s])
        for u in range(h):
            at = pos[s, u, :n].long()
            seen = ((at >= first[s]) & (at > now - 1 - 350))[None].expand(g, n)
            rows_q = q[s, u * g:(u + 1) * g].double()
            x = 10.0 * torch.tanh(rows_q @ k[s, u, :n].double().T / math.sqrt(d) / 10.0)
            w = torch.softmax(x.masked_fill(~seen, -math.inf), -1).nan_to_num(0.0)
            ref = w @ v[s, u, :n].double()
            assert float((outs[1][s, u * g:(u + 1) * g].double() - ref).abs().max()) <= 1e-5 * float(v.abs().max()), (s, u)


def test_calls_that_share_tensor_memory_follow_one_another():
    """The prompt's attention and its compression both take tensor memory: in turn on one stream, and beside each other on two."""
    b, h, g, d, lens = 4, 4, 4, 128, [300, 700, 513, 64]
    q, k, v, plen, mod, kw, _ = prompt_case((b, h, g, d, BF16, lens, "heads"), OPTIONS["cap"], seed=5, junk=False)
    w = torch.randn((d, 16), generator=torch.Generator().manual_seed(3))
    caches = [HashEvictCache(b, h, g, d, 16, [32] * b, w) for _ in range(3)]
    n = q.shape[2]
    work = [c.workspace(n) for c in caches]
    want = caches[0].attend_prompt(q, k, v, plen, mod=mod, out=torch.zeros_like(q))
    caches[0].prefill_compress(q, k, v, plen, n, workspace=work[0])
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(q) for _ in range(2)]
    for _ in range(20):
        caches[1].attend_prompt(q, k, v, plen, mod=mod, out=outs[0], stream=streams[0])
        caches[1].prefill_compress(q, k, v, plen, n, workspace=work[1], stream=streams[0])
        caches[2].prefill_compress(q, k, v, plen, n, workspace=work[2], stream=streams[1])
        caches[2].attend_prompt(q, k, v, plen, mod=mod, out=outs[1], stream=streams[1])
    torch.cuda.synchronize()
    for c, out in zip(caches[1:], outs):
        assert torch.equal(out, want)
        assert torch.equal(c.pos, caches[0].pos) and torch.equal(c.k_cache, caches[0].k_cache)
    assert binding.device_error_count() == 0


def test_outputs_between_other_rows():
    """q, k and v as parts of one projection, outputs into parts of another: what lies between them stays."""
    b, h, g, d, n = 2, 2, 3, 64, 150
    gen = torch.Generator(device="cuda").manual_seed(6)
    fused = torch.randn((b, n, (g + 2) * h, d), generator=gen, device="cuda", dtype=BF16)
    q, k, v = fused.transpose(1, 2).split((g * h, h, h), dim=1)
    cache, plen, rot = make_cache(b, h, g, d, BF16), torch.tensor([n, 77], dtype=torch.int32, device="cuda"), Rotary(d)
    want_q, want_k = cache.rotate_prompt(rot, q.contiguous(), k.contiguous())
    want = cache.attend_prompt(want_q, want_k, v.contiguous(), plen, out=torch.zeros_like(want_q))
    before = fused.clone()
    into = torch.full((b, n, g * h + 1, d), 3.0, device="cuda", dtype=BF16)
    cache.rotate_prompt(rot, q, k, plen, q_out=q, k_out=k)  # in place
    out = into.transpose(1, 2)[:, : g * h]
    assert cache.attend_prompt(q, k, v, plen, out=out) is out
    for s, m in enumerate(plen.tolist()):
        assert torch.equal(out[s, :, :m], want[s, :, :m]) and bool((out[s, :, m:] == 3.0).all())
        assert torch.equal(q[s, :, :m], want_q[s, :, :m]) and torch.equal(fused[s, m:], before[s, m:])
    assert torch.equal(v, before.transpose(1, 2)[:, (g + 1) * h:]) and bool((into[:, :, g * h] == 3.0).all())


def test_offsets_beyond_32_bits():
    """A batch whose last rows lie more than 2^32 elements into q and k."""
    b, h, g, d, n = 2, 1, 1, 128, 300
    far = (2 ** 32 // d + 1000) * d
    base = torch.zeros(far + n * d, device="cuda", dtype=BF16)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = base.as_strided((b, 1, n, d), (far, d * n, d, 1))
    x.copy_(torch.randn((b, 1, n, d), generator=gen, device="cuda"))
    cache, plen = make_cache(b, h, g, d, BF16), torch.tensor([n, n], dtype=torch.int32, device="cuda")
    out = cache.attend_prompt(x, x, x, plen)
    y = x.contiguous()
    assert torch.equal(out, cache.attend_prompt(y, y, y, plen))
    rot = Rotary(d)
    assert torch.equal(cache.rotate_prompt(rot, x, x)[1], cache.rotate_prompt(rot, y, None)[0])


def test_the_binding_refuses():
    cache, rot = make_cache(2, 2, 2, 64, BF16), Rotary(64)
    z = lambda *s, dtype=BF16: torch.zeros(s, device="cuda", dtype=dtype)  # noqa: E731
    q, k, n = z(2, 4, 10, 64), z(2, 2, 10, 64), torch.tensor([10, 10], dtype=torch.int32, device="cuda")
    bad = [
        lambda: cache.rotate_prompt(Rotary(128), q, k), lambda: cache.rotate_prompt(rot, k, k), lambda: cache.rotate_prompt(rot, q.float(), k),
        lambda: cache.rotate_prompt(rot, q, k, n.long()), lambda: cache.rotate_prompt(rot, q, k, positions=n), lambda: cache.rotate_prompt(rot, q.cpu(), k),
        lambda: cache.rotate_prompt(rot, z(2, 4, 10, 128)[..., ::2], k), lambda: cache.rotate_prompt(rot, None, k, q_out=q),
        lambda: cache.rotate_prompt(rot, z(2, 4, 10, 68)[..., 2:66], k),  # rows that are not 16-byte aligned
        lambda: cache.rotate_prompt(rot, None, None), lambda: cache.rotate_step(rot, q, k), lambda: cache.rotate_step(rot, z(2, 4, 64), z(2, 3, 64)),
        lambda: cache.attend_prompt(q, k, k[:, :, :9], n), lambda: cache.attend_prompt(q, k, z(2, 10, 2, 64).transpose(1, 2), n),
        lambda: cache.attend_prompt(q, k, k, n[:1]), lambda: cache.attend_prompt(q, k, k, n, doc_start=n), lambda: cache.attend_prompt(q, k, k, n, prefix_len=n.cpu()),
        lambda: cache.attend_prompt(q, k, k, n, mod=ScoreMod(slopes=torch.ones(3, device="cuda"))), lambda: cache.attend_prompt(q, k, k, n, mod=ScoreMod(window=-2)),
        lambda: cache.attend_prompt(q, k, k, n, out=k), lambda: ScoreMod(slopes=torch.ones(4)), lambda: ScoreMod(slopes=torch.ones(8, device="cuda")[::2]),
        lambda: cache.attend_scored(z(2, 4, 32)), lambda: cache.attend_scored(z(2, 4, 64, dtype=F32)), lambda: cache.attend_scored(z(2, 64, 4).transpose(1, 2)),
        lambda: cache.rotate_prompt(rot, q[0], k[0]), lambda: cache.attend_prompt(q[0], k[0], k[0], n), lambda: cache.rotate_step(rot, None, None),
        lambda: cache.rotate_prompt(rot, q, k, k_out=torch.empty(2, 1, 10, 64, device="cuda", dtype=BF16).expand(2, 2, 10, 64)),
        lambda: cache.attend_scored(z(2, 4, 64), first_pos=n.long()), lambda: cache.attend_scored(z(2, 4, 64), out=z(2, 4, 64)),
    ]
    for i, call in enumerate(bad):
        try:
            call()
        except HashEvictError:
            continue
        pytest.fail(f"call {i} was taken")
    assert binding.device_error_count() == 0
