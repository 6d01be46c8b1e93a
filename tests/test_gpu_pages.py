"""The paged cache: appended rows bit by bit, attention and rows read back against their definitions in 64 bits."""
import math

import pytest
import torch

import page_reference as ref
from layer_reference import attend, tolerance
from paper_2412_16187_b200 import HashEvictError, PagedCache, Rotary, ScoreMod, device_error_count
from test_gpu_layer_ops import BF16, F32, rows

pytestmark = pytest.mark.gpu


def paged(gen, b, h, g, d, p, dtype, eight, most, spare=2, missing=()):
    """A cache of room for `most` tokens a sequence, its pages in no order. missing: (sequence, page) pairs whose entry names no page."""
    per = (most + p - 1) // p
    order = torch.randperm(b * per + spare, generator=gen, device="cuda").to(torch.int32)
    table = order[: b * per].view(b, per).clone()
    for i, (s, at) in enumerate(missing):
        table[s, at] = (-1, b * per + spare, -(2 ** 31), 2 ** 31 - 1)[i % 4]
    return PagedCache(b, h, g, d, table, b * per + spare, p, dtype=dtype, eight_bit=eight)


def poison(cache):
    """What pages hold that nobody wrote: anything (in 8 bits a NaN), to be left alone."""
    for x in (cache.k_pages, cache.v_pages):
        x.view(torch.uint8).fill_(0x7F)
    if cache.eight_bit:
        cache.k_scale.fill_(3.0), cache.v_scale.fill_(math.nan)


def model_of(cache):
    m = {x: None if getattr(cache, x) is None else getattr(cache, x).clone() for x in ("k_pages", "v_pages", "k_scale", "v_scale")}
    return {**m, "page_table": cache.page_table, "length": cache.length}


def same(cache, model):
    for x in ("k_pages", "v_pages"):
        a, b = getattr(cache, x).view(torch.uint8), model[x].view(torch.uint8)
        if cache.eight_bit:  # a NaN is any of its two codes
            a, b = torch.where((a & 127) == 127, 127, a), torch.where((b & 127) == 127, 127, b)
        assert torch.equal(a, b), (x, int((a != b).sum()))
    if cache.eight_bit:
        for x in ("k_scale", "v_scale"):
            assert torch.equal(torch.nan_to_num(getattr(cache, x), nan=-1.0), torch.nan_to_num(model[x], nan=-1.0)), x


def grown(gen, b, h, n, d, dtype, layout):
    """Rows whose size changes from token to token, so that scales of pages grow at any token; an infinity and a NaN, a row of zeros and tiny values among them."""
    x = rows(gen, b, h, n, d, dtype, layout)
    x = x.mul_(torch.exp2(torch.randint(-12, 9, (b, 1, n, 1), generator=gen, device="cuda").to(dtype)))
    x[0, 0, n // 2] = 0.0
    if n > 6:
        x[-1, -1, 3, 1], x[-1, -1, n - 2, 0], x[0, 0, 5, :4] = math.inf, math.nan, 2.0 ** -120
    return x


# (B, H, d, page, dtype, 8 bits, rotated channels (0: none), interleaved, tokens of each call, layout)
APPENDS = [
    (1, 4, 64, 16, F32, False, 64, False, [1, 1, 14, 40], "heads"), (3, 2, 128, 64, BF16, True, 128, False, [100, 1, 1, 61, 200], "tokens"),
    (2, 3, 128, 32, BF16, False, 32, True, [31, 2, 64], "heads"), (2, 8, 128, 128, BF16, True, 0, False, [127, 1, 1, 130], "tokens"),
    (2, 1, 80, 16, BF16, True, 20, False, [5, 60, 17], "heads"), (1, 2, 96, 32, BF16, True, 36, True, [33, 1, 90], "tokens"), (2, 2, 72, 64, BF16, False, 10, False, [70, 1, 3], "heads"),
    (1, 2, 256, 128, BF16, True, 256, False, [300, 1], "heads"), (1, 2, 256, 128, F32, True, 128, False, [130, 1, 5], "tokens"), (2, 2, 64, 64, F32, True, 64, True, [65, 1, 62, 1], "heads"),
    (1, 33, 128, 64, BF16, True, 128, False, [640], "tokens"), (1, 1, 128, 64, F32, False, 126, False, [66, 1], "heads"), (2, 2, 16, 16, BF16, True, 6, False, [17, 30, 1], "heads"),
    (1, 3, 128, 128, F32, False, 128, False, [129, 1, 300], "heads"), (1, 1, 8, 16, BF16, False, 8, False, [20], "heads"),
    (2, 2, 128, 16, BF16, True, 100, True, [40, 1, 30], "tokens"), (1, 2, 72, 16, BF16, False, 72, True, [20, 1], "heads"), (1, 5, 80, 128, F32, True, 60, True, [130, 1], "heads"),
    (1, 2, 256, 128, BF16, True, 200, True, [200, 2], "tokens"), (1, 9, 128, 128, BF16, True, 128, True, [300, 7], "tokens"),
]


@pytest.mark.parametrize("b, h, d, p, dtype, eight, r, inter, calls, layout", APPENDS, ids=lambda x: str(x) if isinstance(x, (int, str)) else None)
def test_append(b, h, d, p, dtype, eight, r, inter, calls, layout):
    """Chunk by chunk, ragged, the pages are those of the definition, bit for bit, and no other byte of theirs is touched."""
    gen = torch.Generator(device="cuda").manual_seed(d * 7 + p)
    cache = paged(gen, b, h, 2, d, p, dtype, eight, sum(calls) + p)
    poison(cache)
    model = model_of(cache)
    rot = Rotary(d, r, base=10000.0, interleaved=inter, scaling={"kind": "yarn", "factor": 4.0, "length": 2048}) if r else None
    for i, n in enumerate(calls):
        k, v = (grown(gen, b, h, n, d, dtype, layout) for _ in "kv")
        new = None if i == 0 else torch.tensor([n] + [max(n - 1 - s, 0) for s in range(b - 1)], dtype=torch.int32, device="cuda")
        cache.length += n if new is None else new
        pos = (cache.length - (n if new is None else new))[:, None] + torch.arange(n, dtype=torch.int32, device="cuda")
        turned = k if rot is None else cache.rotate_prompt(rot, None, k, positions=pos.contiguous())[1]
        cache.append(k, v, new, rotary=rot)
        ref.append(model, (turned, v), new)
        same(cache, model)
        cache.append(k, v, new, rotary=rot)  # once more: nothing changes
        same(cache, model)


def test_a_prompt_appended_at_once_or_token_by_token():
    """Rows whose codes are all normal numbers give the same pages whichever way they come."""
    b, h, d, p, n = 2, 2, 64, 32, 75
    gen = torch.Generator(device="cuda").manual_seed(3)
    once, step = (paged(torch.Generator(device="cuda").manual_seed(4), b, h, 1, d, p, BF16, True, n) for _ in "12")
    k, v = (torch.randn((b, h, n, d), generator=gen, device="cuda").sign() * (1 + torch.rand((b, h, n, d), generator=gen, device="cuda") * 100) for _ in "kv")
    k, v, rot = k.to(BF16), v.to(BF16), Rotary(d, 32)
    once.length += n
    once.append(k, v, rotary=rot)
    turned = once.rotate_prompt(rot, None, k)[1].float().abs()
    assert float(turned.amax()) < 448
    for t in range(n):
        step.length += 1
        step.append(k[:, :, t:t + 1], v[:, :, t:t + 1], rotary=rot)
    assert torch.equal(once.k_scale, step.k_scale) and torch.equal(once.v_scale, step.v_scale)
    assert torch.equal(once.v_pages.view(torch.uint8), step.v_pages.view(torch.uint8))
    big = once.k_pages.float().abs() >= 2.0 ** -6
    assert torch.equal(once.k_pages.view(torch.uint8)[big], step.k_pages.view(torch.uint8)[big])
    assert bool(((once.k_pages.float() - step.k_pages.float()).abs() <= 2.0 ** -10 * 9).all())  # a page's scale grows over 2^9 at most: 2^-10 each time


@pytest.mark.parametrize("eight", [False, True])
def test_rows_that_have_no_place_are_dropped(eight):
    b, h, d, p = 4, 2, 32, 16
    gen = torch.Generator(device="cuda").manual_seed(9)
    cache = paged(gen, b, h, 1, d, p, BF16, eight, 48, missing=((1, 0), (1, 1), (2, 2), (3, 1)))
    poison(cache)
    model = model_of(cache)
    k, v = (rows(gen, b, h, 70, d, BF16) for _ in "kv")
    for held, new in (([70, 48, 60, 33], [70, 40, 20, 33]), ([5, -3, 2 ** 31 - 1, 49], [70, 4, 70, 1]), ([0, 10, 50, 48], [3, -5, 2 ** 31 - 1, 0]), ([20, 0, 16, 47], [2 ** 30, 0, 16, 47])):
        cache.length.copy_(torch.tensor(held))
        lens = torch.tensor(new, dtype=torch.int32, device="cuda")
        cache.append(k, v, lens)
        ref.append(model, (k, v), lens)
        same(cache, model)
    cache.append(k[:, :, :0], v[:, :, :0])
    same(cache, model)


def test_largest_and_smallest_values():
    """Scales at the ends of their range: the largest numbers of fp32 and bf16, numbers below what 2^-100 can hold, subnormal ones, zeros."""
    for dtype in (BF16, F32):
        gen = torch.Generator(device="cuda").manual_seed(5)
        cache = paged(gen, 1, 1, 1, 16, 16, dtype, True, 16 * 12)
        poison(cache)
        model = model_of(cache)
        x = torch.randn((1, 1, 16 * 12, 16), generator=gen, device="cuda").sign()
        for at, size in enumerate((torch.finfo(dtype).max, 2.0 ** 127, 448.0, 449.0, 448.0 * 2 ** 20, 2.0 ** -90, 448 * 2.0 ** -100, 2.0 ** -106, 2.0 ** -126, 2.0 ** -133, 0.0, 1.75)):
            x[:, :, 16 * at: 16 * at + 16] *= size
        x = x.to(dtype)
        cache.length += 16 * 12
        cache.append(x, x.flip(2))
        ref.append(model, (x, x.flip(2)), None)
        same(cache, model)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d, p", [(128, 64), (256, 128)])
def test_a_page_that_came_with_another_scale(dtype, d, p):
    """Rows join a page whose scale is no power of two and large enough for them: it stays, as do the rows that are there, and each new entry is off by half a step at most."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    cache = paged(gen, 1, 2, 1, d, p, dtype, True, p)
    k, v = (rows(gen, 1, 2, p, d, dtype) for _ in "kv")
    k[0, 1, p - 1, 3], v[0, 0, 9, 0] = math.inf, math.nan
    cache.length += 5
    cache.append(k[:, :, :5], v[:, :, :5])
    page = int(cache.page_table[0, 0])
    for x in (cache.k_scale, cache.v_scale):
        x[page] = 0.3
    old = [x[page, :, :5].view(torch.uint8).clone() for x in (cache.k_pages, cache.v_pages)]
    cache.length += p - 5
    cache.append(k[:, :, 5:], v[:, :, 5:])
    for x, pages, scale, was in ((k, cache.k_pages, cache.k_scale, old[0]), (v, cache.v_pages, cache.v_scale, old[1])):
        assert bool((scale[page] == torch.tensor(0.3, device="cuda")).all()) and torch.equal(pages[page, :, :5].view(torch.uint8), was)
        want, got = x[0, :, 5:].double(), pages[page, :, 5:].float().double() * scale[page].double()[:, None, None]
        whole = torch.isfinite(want)
        assert torch.equal(torch.isnan(got), ~whole)
        # half a step of e4m3, and two roundings in fp32 (of 1 / s and of the product) ahead of it
        most = torch.maximum(want.abs() * (2.0 ** -4 + 2.0 ** -20), torch.full_like(want, 0.3 * 2.0 ** -10 * (1 + 2.0 ** -20)))
        assert bool(((got - want).abs() <= most)[whole].all())


def filled(gen, b, h, g, d, p, dtype, eight, lens, missing=(), most=None):
    """A cache that holds `lens` tokens a sequence; what lies behind them is poisoned."""
    cache = paged(gen, b, h, g, d, p, dtype, eight, max(max(lens), 1) if most is None else most, missing=missing)
    poison(cache)
    n = max(max(lens), 1)
    k, v = rows(gen, b, h, n, d, dtype) * 2, rows(gen, b, h, n, d, dtype) * torch.exp2(torch.randint(-3, 4, (b, 1, n, 1), generator=gen, device="cuda").to(dtype))
    cache.length.copy_(torch.tensor(lens))
    for at in range(0, n, 97):  # (several calls: scales of their own history)
        part = cache.length.clamp(max=at + 97)
        new = part - part.clamp(max=at)
        keep = cache.length.clone()
        cache.length.copy_(part)
        first = min(97, n - at)
        sl_k, sl_v = k[:, :, at:at + first], v[:, :, at:at + first]
        cache.append(sl_k, sl_v, new)
        cache.length.copy_(keep)
    return cache


def check_attend(got, cache, q, opt, slopes, first):
    model, g = model_of(cache), cache.G
    for s in range(cache.B):
        n = int(cache.length[s])
        if n == 0:
            assert not got[s].any()
            continue
        k, v = ref.values(model, "k", s, n), ref.values(model, "v", s, n)
        at = torch.arange(n, device="cuda")
        seen = at > n - 1 - opt["window"] if opt.get("window") else torch.ones_like(at, dtype=torch.bool)
        if first is not None:
            seen = seen & (at >= first[s])
        for u in range(cache.H):
            sl = slice(u * g, u * g + g)
            want = attend(q[s, sl][:, None], k[u], v[u], torch.tensor([n - 1], device="cuda"), at, seen[None], opt.get("scale", 0.0), opt.get("cap", 0.0),
                          None if slopes is None else slopes[sl])[:, 0]
            if not seen.any():
                assert not got[s, sl].any()
                continue
            tol = tolerance(want, v[u][seen].abs().max(), F32, True)
            assert bool(((got[s, sl].double() - want).abs() <= tol).all()), (s, u, float((got[s, sl].double() - want).abs().max()))


OPTS = {"plain": {}, "cap": {"cap": 20.0}, "bias": {"slopes": True}, "window": {"window": 33}, "first": {"first": 600}, "window of one": {"window": 1},
        "all": {"cap": 8.0, "slopes": True, "window": 200, "first": 300, "scale": 0.25}, "nothing seen": {"first": 5000}}
CACHES = [
    ((1, 4, 1, 64, 16, F32, False), [128]), ((3, 2, 4, 128, 64, BF16, True), [1, 33, 500]), ((3, 2, 7, 256, 32, BF16, False), [5, 0, 90]), ((2, 2, 3, 48, 16, F32, True), [1, 130]),
    ((1, 8, 4, 128, 128, BF16, True), [2900]), ((2, 1, 8, 64, 32, BF16, True), [700, 64]), ((2, 2, 5, 96, 16, BF16, True), [333, 32]), ((200, 1, 2, 64, 16, BF16, False), list(range(200))),
    ((2, 2, 2, 24, 16, BF16, False), [100, 31]), ((2, 1, 1, 80, 64, BF16, True), [1300, 1]), ((4, 2, 4, 128, 32, BF16, False), [1, 4100, 0, 31]), ((2, 3, 8, 128, 16, BF16, True), [17, 1500]),
    ((1, 2, 2, 256, 128, F32, True), [700]), ((2, 2, 8, 128, 64, F32, True), [600, 63]), ((1, 1, 1, 8, 16, F32, False), [40]), ((300, 2, 4, 64, 32, BF16, True), [7 * i % 97 for i in range(300)]),
    ((3, 2, 4, 64, 128, BF16, False), [2000, 129, 3]), ((2, 1, 6, 104, 16, BF16, False), [900, 15]), ((2, 2, 3, 144, 32, BF16, True), [200, 70]), ((1, 1, 8, 240, 64, F32, True), [150]),
]
NAMES = [f"{'x'.join(map(str, s[:4]))}-p{s[4]}-{'bf16' if s[5] == BF16 else 'fp32'}{'-8bit' if s[6] else ''}-{max(n)}" for s, n in CACHES]


@pytest.mark.parametrize("opt", list(OPTS))
@pytest.mark.parametrize("shape, lens", CACHES, ids=NAMES)
def test_attend(shape, lens, opt):
    b, h, g, d, p, dtype, eight = shape
    gen = torch.Generator(device="cuda").manual_seed(d + b)
    o = OPTS[opt]
    cache = filled(gen, b, h, g, d, p, dtype, eight, lens)
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    slopes = torch.exp2(-torch.arange(1, h * g + 1, device="cuda") * 8.0 / (h * g)) if o.get("slopes") else None
    first = torch.tensor([n * o["first"] // 1000 for n in lens], dtype=torch.int32, device="cuda") if "first" in o else None
    mod = ScoreMod(scale=o.get("scale", 0.0), softcap=o.get("cap", 0.0), window=o.get("window", 0), slopes=slopes)
    got = cache.attend(q, mod, first_pos=first)
    check_attend(got, cache, q, o, slopes, first)
    kept = torch.full((cache.workspace().numel(),), 255, dtype=torch.uint8, device="cuda")  # whatever the workspace holds, the result is the same, bit for bit
    assert torch.equal(cache.attend(q, mod, first_pos=first, workspace=kept), got) and torch.equal(cache.attend(q, mod, first_pos=first, workspace=kept), got)
    assert device_error_count() == 0


@pytest.mark.parametrize("shape, lens", [CACHES[i] for i in (1, 4, 7, 10, 13)], ids=[NAMES[i] for i in (1, 4, 7, 10, 13)])
def test_pages_that_are_not_there_read_as_zeros(shape, lens):
    b, h, g, d, p, dtype, eight = shape
    gen = torch.Generator(device="cuda").manual_seed(d)
    gone = [(s, a) for s, n in enumerate(lens) for a in range(0, (n + p - 1) // p, 3)][:9]
    cache = filled(gen, b, h, g, d, p, dtype, eight, lens, missing=gone)
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    check_attend(cache.attend(q), cache, q, {}, None, None)
    k, v = cache.read(max(lens))
    model = model_of(cache)
    for s, n in enumerate(lens):
        if n:
            assert torch.equal(k[s, :, :n].double(), ref.values(model, "k", s, n)) and torch.equal(v[s, :, :n].double(), ref.values(model, "v", s, n))


@pytest.mark.parametrize("shape, lens", CACHES, ids=NAMES)
def test_read(shape, lens):
    b, h, g, d, p, dtype, eight = shape
    gen = torch.Generator(device="cuda").manual_seed(d + 1)
    cache = filled(gen, b, h, g, d, p, dtype, eight, lens)
    model, n = model_of(cache), max(lens)
    for m, first, layout in ((n, None, "heads"), (n // 2 + 1, [x // 3 for x in lens], "tokens"), (3, [-7 if s % 2 else 2 ** 31 - 1 for s in range(b)], "heads")):
        k, v = (torch.full_like(rows(gen, b, h, m, d, dtype, layout), 7.0) for _ in "kv")
        if layout == "tokens":
            k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
        start = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
        cache.read(m, start, k_out=k, v_out=v)
        for s, held in enumerate(lens):
            at = 0 if first is None else max(first[s], 0)
            some = max(min(held - at, m), 0)
            for x, y in (("k", k), ("v", v)):
                assert bool((y[s, :, some:] == 7.0).all())
                if some:
                    assert torch.equal(y[s, :, :some].double(), ref.values(model, x, s, held)[:, at:at + some])
        only = torch.full_like(k, 7.0)
        cache.read(m, start, v_out=only)
        assert torch.equal(only, v)


def test_scales_that_are_no_powers_of_two_are_taken():
    gen = torch.Generator(device="cuda").manual_seed(2)
    cache = filled(gen, 2, 2, 4, 128, 32, BF16, True, [300, 95])
    cache.k_scale *= torch.rand(cache.k_scale.shape, generator=gen, device="cuda") + 0.5
    cache.v_scale *= 1.1
    q = torch.randn((2, 8, 128), generator=gen, device="cuda", dtype=BF16)
    check_attend(cache.attend(q), cache, q, {}, None, None)
    k, _ = cache.read(300)
    want = ref.values(model_of(cache), "k", 0, 300)
    assert bool(((k[0].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all())


@pytest.mark.parametrize("shape, lens", [CACHES[i] for i in (0, 1, 4, 6, 10)], ids=[NAMES[i] for i in (0, 1, 4, 6, 10)])
def test_what_is_no_number_reaches_those_who_see_it(shape, lens):
    b, h, g, d, p, dtype, eight = shape
    gen = torch.Generator(device="cuda").manual_seed(8)
    cache = filled(gen, b, h, g, d, p, dtype, eight, lens)
    s = max(range(b), key=lambda i: lens[i])
    n, u = lens[s], h - 1
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    first = torch.zeros((b,), dtype=torch.int32, device="cuda")
    first[s] = n // 2 + 1
    clean = cache.attend(q, first_pos=first)
    page, row = int(cache.page_table[s, (n // 2) // p]), (n // 2) % p
    for pages in (cache.k_pages, cache.v_pages):
        if eight:
            pages.view(torch.uint8)[page, u, row, 3] = 0x7F
        else:
            pages[page, u, row, 3] = math.inf
    assert torch.equal(cache.attend(q, first_pos=first), clean)  # hidden
    got = cache.attend(q)
    assert bool(torch.isnan(got[s, u * g:]).all() if eight else ~torch.isfinite(got[s, u * g:, 3]).any())
    q[s, 0, 5] = math.nan
    got = cache.attend(q, first_pos=first)
    assert bool(torch.isnan(got[s, 0]).all())
    others = torch.ones(got.shape[:2], dtype=torch.bool, device="cuda")
    others[s, 0] = False
    assert torch.equal(got[others], clean[others])


def test_calls_on_other_streams_and_captured_ones_give_the_same_bits():
    b, h, g, d, p, lens = 3, 2, 4, 128, 32, [900, 40, 333]
    gen = torch.Generator(device="cuda").manual_seed(6)
    caches = [filled(torch.Generator(device="cuda").manual_seed(6), b, h, g, d, p, BF16, True, lens, most=1024) for _ in "1234"]
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=BF16)
    k, v = (rows(gen, b, h, 1, d, BF16) for _ in "kv")
    rot, mod = Rotary(d), ScoreMod(softcap=30.0, window=500)

    def step(cache, stream):
        cache.append(k, v, rotary=rot, stream=stream)
        return cache.attend(q, mod, stream=stream), *cache.read(1024, stream=stream)

    for c in caches:
        c.length += 1
    torch.cuda.synchronize()
    want = [x.clone() for x in step(caches[0], None)]
    streams, got, graphs = [torch.cuda.Stream() for _ in range(3)], [], []
    for c, st in zip(caches[1:3], streams):
        got.append(step(c, st))
    st = streams[2]
    with torch.cuda.stream(st):
        step(caches[3], st)
        st.synchronize()
        for _ in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=st):
                got.append(step(caches[3], st))
    for graph in graphs:
        graph.replay(), graph.replay()
    torch.cuda.synchronize()
    for out in got:
        assert torch.equal(out[0], want[0])
        for s, n in enumerate(lens):
            for x, y in zip(out[1:], want[1:]):
                assert torch.equal(x[s, :, : n + 1], y[s, :, : n + 1])


def test_offsets_beyond_32_bits():
    """Pages behind the first 2^31 bytes and elements of a pool; rows that lie as far apart."""
    h, d, p = 8, 128, 128
    n_pages = 2 ** 32 // (h * p * d) + 40  # 2^32 codes each for K and V
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2, 1], [n_pages // 2 + 1, n_pages - 5, 0, 2]], dtype=torch.int32, device="cuda")
    for eight in (True, False):
        if not eight:
            n_pages = n_pages // 2 + 20
            table = table.clamp(max=n_pages - 1) - torch.tensor([[0, 0, 1, 0], [0, 4, 0, 0]], dtype=torch.int32, device="cuda")
        cache = PagedCache(2, h, 2, d, table, n_pages, p, dtype=BF16, eight_bit=eight)
        n = 4 * p - 9
        k, v = (rows(gen, 2, h, n, d, BF16) for _ in "kv")
        cache.length.copy_(torch.tensor([n, n - 70]))
        cache.append(k, v, cache.length)
        q = torch.randn((2, h * 2, d), generator=gen, device="cuda", dtype=BF16)
        got = cache.attend(q)
        used = table.flatten().long()
        small = PagedCache(2, h, 2, d, torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4), 8, p, dtype=BF16, eight_bit=eight, length=cache.length)
        for x in ("k_pages", "v_pages") + (("k_scale", "v_scale") if eight else ()):
            src, dst = getattr(cache, x), getattr(small, x)
            dst.view(torch.uint8).copy_(src.view(torch.uint8)[used]) if x.endswith("pages") else dst.copy_(src[used])
        model = {**model_of(small), "k_pages": torch.zeros_like(small.k_pages), "v_pages": torch.zeros_like(small.v_pages)}
        ref.append(model, (k, v), cache.length)
        same(small, model)
        assert torch.equal(small.attend(q), got)
        for x, y in zip(cache.read(n), small.read(n)):
            assert torch.equal(x[0, :, :n], y[0, :, :n]) and torch.equal(x[1, :, : n - 70], y[1, :, : n - 70])
        del cache, small
    far = torch.empty((2, 1, 40, 2 ** 26), dtype=BF16, device="cuda")[..., :128]  # rows 2^26 elements apart
    k = rows(gen, 2, 1, 40, 128, BF16)
    far.copy_(k)
    cache = paged(gen, 2, 1, 1, 128, 16, BF16, False, 40)
    cache.length += 40
    cache.append(far, far)
    assert torch.equal(cache.read(40)[0], k)
    far.zero_()
    cache.read(40, k_out=far)
    assert torch.equal(far, k)


def test_the_binding_refuses():
    b, h, g, d, p = 2, 2, 2, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = paged(gen, b, h, g, d, p, BF16, False, 64)
    k, q = rows(gen, b, h, 3, d, BF16), torch.zeros((b, h * g, d), dtype=BF16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    for call in (lambda: cache.append(k, k[:, :, :2]), lambda: cache.append(k.float(), k.float()), lambda: cache.append(k, k.transpose(1, 2).contiguous().transpose(1, 2)),
                 lambda: cache.append(k, k, torch.zeros((b,), device="cuda")), lambda: cache.append(k, k, torch.zeros((b + 1,), **i32)), lambda: cache.append(k.cpu(), k.cpu()),
                 lambda: cache.append(k, k, rotary=Rotary(128)), lambda: cache.append(k[:1], k[:1]), lambda: cache.attend(q.float()), lambda: cache.attend(q[:1]),
                 lambda: cache.attend(q, out=torch.zeros_like(q)), lambda: cache.attend(q, first_pos=torch.zeros((b, 1), **i32)),
                 lambda: cache.attend(q, ScoreMod(slopes=torch.zeros((3,), device="cuda"))), lambda: cache.attend(q, workspace=torch.zeros((4, 4), dtype=torch.uint8, device="cuda")),
                 lambda: cache.read(4, k_out=k), lambda: cache.read(3, k_out=k, v_out=k), lambda: cache.read(3, torch.zeros((b,), device="cuda"), k_out=k), lambda: cache.read(-1),
                 lambda: PagedCache(b, h, g, d, torch.zeros((b, 4), dtype=torch.int64, device="cuda"), 4), lambda: PagedCache(b, h, g, d, torch.zeros((3, 4), **i32), 4),
                 lambda: PagedCache(b, h, g, d, torch.zeros((b, 4), dtype=torch.int32), 4), lambda: PagedCache(b, h, g, d, torch.zeros((b, 4), **i32), 4, length=torch.zeros((b,), device="cuda")),
                 lambda: PagedCache(b, h, g, 72, torch.zeros((b, 4), **i32), 4, eight_bit=True).attend(torch.zeros((b, h * g, 72), dtype=BF16, device="cuda")),
                 lambda: PagedCache(b, h, g, d, torch.zeros((b, 4), **i32), 4, page_size=48).attend(q)):
        with pytest.raises((HashEvictError, RuntimeError)):
            call()
    expanded = k[:, :1].expand(b, h, 3, d)
    cache.length += 3
    cache.append(expanded, expanded)  # inputs may be one tensor seen several times, outputs not
    assert torch.equal(cache.read(3)[1], expanded)
    with pytest.raises(HashEvictError, match="overlap"):
        cache.read(3, k_out=expanded)
