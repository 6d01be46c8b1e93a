"""Values that are not finite in a prompt: what rows see reaches them, what they do not see does not, and the call takes about as long as ever."""
import math

import pytest
import torch

from layer_reference import prompt_seen
from paper_2412_16187_b200 import ScoreMod
from test_gpu_layer_ops import BF16, F32, make_cache, rows

pytestmark = pytest.mark.gpu


def least_time(call):
    for _ in range(2):
        call()
    times = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


def prompt(dtype, d, n, heads=8, group=4):
    gen = torch.Generator(device="cuda").manual_seed(d + n)
    cache = make_cache(1, heads // group, group, d, dtype)
    q, k, v = rows(gen, 1, heads, n, d, dtype), rows(gen, 1, heads // group, n, d, dtype), rows(gen, 1, heads // group, n, d, dtype)
    return cache, q, k, v, torch.tensor([n], dtype=torch.int32, device="cuda")


SHAPES = [(BF16, 128, 4096), (BF16, 64, 4096), (BF16, 128, 600), (BF16, 200, 700), (F32, 64, 2048), (F32, 128, 300)]


@pytest.mark.parametrize("dtype, d, n", SHAPES)
@pytest.mark.parametrize("what", ["key 0", "key -inf", "value 0", "value inf", "all values", "a query", "late value"])
def test_what_is_not_finite_costs_little(dtype, d, n, what):
    """About as long as on finite rows: a row that sees a NaN is one whatever is done."""
    cache, q, k, v, plen = prompt(dtype, d, n)
    out, mod = torch.empty_like(q), ScoreMod(window=n // 2) if what == "late value" else None
    call = lambda: cache.attend_prompt(q, k, v, plen, mod=mod, out=out)  # noqa: E731
    usual = least_time(call)
    assert bool(torch.isfinite(out).all())
    clean = out.clone()
    bad = torch.zeros((n, d), dtype=torch.bool, device="cuda")  # where outputs of the first KV head's queries are no numbers
    g, sees = q.shape[1] // k.shape[1], prompt_seen(n, n // 2 if what == "late value" else 0)
    if what == "key 0":
        k[0, 0, 0, 7] = math.nan
        bad[:] = True
    elif what == "key -inf":  # a score of +inf or -inf: a row with the first is no number, one with the second does not weigh the key
        k[0, 0, 0, 7] = math.inf
        q[0, :g, :, 7] = 1.0
        bad[:] = True
    elif what == "value 0":
        v[0, 0, 0, 7] = math.nan
        bad[:, 7] = True
    elif what == "value inf":
        v[0, 0, 0, 7] = math.inf
    elif what == "all values":
        v[0, 0] = math.nan
        bad[:] = True
    elif what == "a query":
        q[0, 1, n // 2] = math.nan
    else:
        v[0, 0, n // 3, 5] = math.nan
        bad[:, 5] = sees[:, n // 3]
    took = least_time(call)
    assert torch.equal(out[0, g:], clean[0, g:])
    if what == "a query":
        same = torch.ones(out.shape[1:3], dtype=torch.bool, device="cuda")
        same[1, n // 2] = False
        assert bool(torch.isnan(out[0, 1, n // 2]).all()) and torch.equal(out[0][same], clean[0][same])
    elif what == "value inf":  # (0 * inf where a weight underflows)
        assert not bool(torch.isfinite(out[0, :g, :, 7]).any())
        others = [c for c in range(d) if c != 7]
        assert torch.equal(out[0, :g][:, :, others], clean[0, :g][:, :, others])
    else:
        assert torch.equal(torch.isnan(out[0, :g]), bad.expand(g, n, d))
    # (a window lets one tile of rows a head out of sight of the NaN: those rows are computed anew)
    assert took <= (400 if what == "late value" else 10) * usual, (took, usual)


@pytest.mark.parametrize("dtype, d, n", [(BF16, 128, 700), (BF16, 64, 500), (BF16, 136, 400), (F32, 64, 300)])
def test_seen_and_hidden_values_that_are_not_finite_together(dtype, d, n):
    """A tile in which rows hide some of what is not finite and see the rest: each has exactly what it sees."""
    cache, q, k, v, plen = prompt(dtype, d, n, heads=2, group=2)
    doc = torch.where(torch.arange(n, device="cuda") < n // 2 + 9, 0, n // 2 + 9).to(torch.int32)[None].contiguous()
    spots = [(3, 1, math.nan), (n // 2, 2, math.inf), (n // 2 + 20, 3, math.nan), (n // 2 + 21, 3, math.inf), (n - 40, 4, -math.inf), (n - 30, 4, math.inf), (n - 2, 6, math.nan)]
    for window in (0, 100):
        out = {}
        for name in ("with", "without"):
            x = v.clone()
            if name == "with":
                for j, c, value in spots:
                    x[0, 0, j, c] = value
            else:
                for j, c, _ in spots:
                    x[0, 0, j, c] = 0.0
            out[name] = cache.attend_prompt(q, k, x, plen, mod=ScoreMod(window=window), doc_start=doc)
        sees = prompt_seen(n, window, doc[0])
        want = torch.zeros((n, d), dtype=torch.float64, device="cuda")
        for j, c, value in spots:  # inf + -inf and anything + NaN are NaN
            want[:, c] += torch.where(sees[:, j], value, 0.0)
        got = out["with"][0].double()
        touched = want != 0  # (NaN too)
        assert torch.equal(torch.isnan(got)[:, torch.isnan(want)], torch.ones_like(torch.isnan(got)[:, torch.isnan(want)]))
        rest = touched & ~torch.isnan(want)
        assert bool((got[:, rest] == want[rest]).all())
        # elsewhere: both within the tolerance of exact arithmetic, which rows computed again meet with fp32 weights
        near = (got - out["without"][0].double()).abs()[:, ~touched]
        assert float(near.max()) <= 2 * (2.0 ** -8 + 2.0 ** -8 + 2e-5) * float(v.abs().max())


@pytest.mark.parametrize("dtype, d, n", SHAPES)
@pytest.mark.parametrize("mask", ["plain", "cap", "slopes", "window"])
@pytest.mark.parametrize("group", [4, 1])
def test_padding_ahead_of_a_prompt_may_hold_anything(dtype, d, n, mask, group):
    """Padded on the left: padding sees nothing and nobody sees it. Nothing of it is ever multiplied, so the call costs what it always does."""
    cache, q, k, v, _ = prompt(dtype, d, n, heads=8 if group > 1 else 3, group=group)
    cache2 = make_cache(2, k.shape[1], group, d, dtype)
    q, k, v = (x.expand(2, -1, -1, -1).clone() for x in (q, k, v))
    pads = [37, n // 3 + 1]
    at = torch.arange(n, device="cuda")
    doc = torch.stack([torch.where(at < p, 2 ** 30, p) for p in pads]).to(torch.int32)
    plen = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    heads = q.shape[1]
    mod = {"plain": None, "cap": ScoreMod(softcap=20.0), "slopes": ScoreMod(slopes=torch.full((heads,), 0.1, device="cuda")), "window": ScoreMod(window=101)}[mask]
    out = torch.empty_like(q)
    call = lambda: cache2.attend_prompt(q, k, v, plen, mod=mod, doc_start=doc, out=out)  # noqa: E731
    usual = least_time(call)
    clean = out.clone()
    assert bool(torch.isfinite(clean).all()) and not clean[0, :, :37].any()
    for s, p in enumerate(pads):
        q[s, :, :p], k[s, :, :p], v[s, :, :p] = math.inf, math.nan, math.nan
    out.fill_(7.0)
    took = least_time(call)
    assert torch.equal(out, clean)
    assert took <= 10 * usual, (took, usual)


@pytest.mark.parametrize("dtype, d, n", SHAPES)
@pytest.mark.parametrize("mod", [None, ScoreMod(window=200)])
def test_prompt_scores_of_minus_infinity_have_no_weight(dtype, d, n, mod):
    """Keys of the first half at -inf: rows that see them alone give zeros, the others what they would give without them."""
    cache, q, k, v, plen = prompt(dtype, d, n)
    g, half = q.shape[1] // k.shape[1], n // 2 + 3
    q[0, :g, :, 3] = 1.0
    out = cache.attend_prompt(q, k, v, plen, mod=mod)
    doc = torch.full((1, n), half, dtype=torch.int32, device="cuda")
    want = cache.attend_prompt(q, k, v, plen, mod=mod, doc_start=doc)
    k[0, 0, :half, 3] = -math.inf
    got = cache.attend_prompt(q, k, v, plen, mod=mod)
    assert torch.equal(got[0, g:], out[0, g:])
    assert not got[0, :g, :half].any()
    # both within the tolerance of exact arithmetic: weights and outputs rounded to bf16 where they are
    limit = (2 * 2e-5 + (2.0 ** -7 if dtype == BF16 and d <= 128 else 0.0) + (2.0 ** -7 if dtype == BF16 else 0.0)) * float(v[0, 0].abs().max())
    assert float((got[0, :g, half:].double() - want[0, :g, half:].double()).abs().max()) <= limit
