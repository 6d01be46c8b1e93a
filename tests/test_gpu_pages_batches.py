"""Attention over pages for padded and for large batches: sequences that see nothing beside others, more sequences than a CTA has threads."""
import pytest
import torch

from layer_reference import tolerance
from paper_2412_16187_b200 import ScoreMod, device_error_count
from test_gpu_layer_ops import BF16, F32, make_cache, rows
from test_gpu_pages import check_attend, filled

pytestmark = pytest.mark.gpu


def nan_out(cache):
    return torch.full((cache.B, cache.H * cache.G, cache.d), torch.nan, device="cuda")


# B, H, G, d, page, dtype, 8 bits, lengths
PADDED = [
    (7, 32, 8, 128, 64, BF16, True, [0, 0, 300, 0, 5, 200, 0]), (5, 16, 4, 128, 32, BF16, False, [0, 100, 0, 0, 0]), (160, 2, 3, 80, 16, BF16, True, [i % 3 * (i % 50) for i in range(160)]),
    (200, 4, 1, 64, 128, F32, True, [0] * 200), (150, 1, 8, 16, 16, BF16, False, [0] * 149 + [40]),
]


@pytest.mark.parametrize("b, h, g, d, p, dtype, eight, lens", PADDED, ids=lambda x: str(x) if isinstance(x, int) else None)
def test_sequences_that_see_nothing_give_zeros(b, h, g, d, p, dtype, eight, lens):
    gen = torch.Generator(device="cuda").manual_seed(b)
    cache = filled(gen, b, h, g, d, p, dtype, eight, lens)
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    out = nan_out(cache)
    cache.attend(q, out=out)
    check_attend(out, cache, q, {}, None, None)
    first = torch.tensor([n // 2 if s % 2 else n + s for s, n in enumerate(lens)], dtype=torch.int32, device="cuda")  # and those whose tokens are all hidden
    out = nan_out(cache)
    cache.attend(q, ScoreMod(window=90), first_pos=first, out=out)
    check_attend(out, cache, q, {"window": 90}, None, first)
    cache.length.sub_(2 ** 30)  # negative ones hold nothing
    out = nan_out(cache)
    cache.attend(q, out=out)
    assert not out.any() and device_error_count() == 0


def test_rows_of_sequences_without_rows_or_keys():
    """One row a sequence over other keys: without keys zeros, without a row nothing is written."""
    b, h, g, d, m = 170, 4, 4, 64, 60
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = rows(gen, b, h * g, 1, d, BF16), rows(gen, b, h, m, d, BF16), rows(gen, b, h, m, d, BF16)
    ql, kl = (torch.tensor([i % c for i in range(b)], dtype=torch.int32, device="cuda") for c in (2, 3))
    cache = make_cache(b, h, g, d, BF16)
    out = cache.attend_cross(q, k, v, ql, kl, out=torch.full_like(q, torch.nan), workspace=cache.cross_workspace(1, m))
    assert bool(torch.isnan(out[ql == 0]).all()) and not out[(ql == 1) & (kl == 0)].any()
    one, two = (ql == 1) & (kl == 1), (ql == 1) & (kl == 2)
    assert torch.equal(out[one], v[one][:, :, :1].repeat_interleave(g, 1))
    s = (q[two].double().view(-1, h, g, d) @ k[two][:, :, :2].double().mT / d ** 0.5).softmax(-1)
    want = (s @ v[two][:, :, :2].double()).view(-1, h * g, 1, d)
    assert bool(((out[two].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2e-5 * float(v.abs().max())).all())
    assert device_error_count() == 0


# More sequences than a CTA has threads (256 for bf16 pages, 384 and 512 for codes of more and of up to 64 channels): a thread counts several, runs of empty ones among them
# at the start, inside and at the end of what it counts.
MANY = [
    (257, 1, 2, 128, 16, BF16, False, lambda s: 1 + s % 37), (700, 2, 4, 64, 32, BF16, False, lambda s: 0 if s < 300 or 340 < s < 500 or s > 690 else s % 90), (385, 1, 4, 128, 64, BF16, True, lambda s: s % 70 if s % 2 else 0),
    (1100, 1, 8, 128, 16, BF16, True, lambda s: 0 if s % 3 < 2 else s % 60), (513, 2, 1, 64, 16, BF16, True, lambda s: 3), (1600, 1, 3, 48, 32, F32, True, lambda s: 0 if s % 4 in (0, 3) else s % 50),
    (600, 1, 1, 64, 16, BF16, True, lambda s: 700 if s == 599 else 0), (2000, 1, 2, 32, 16, BF16, False, lambda s: 40 * (s % 7 == 6)),
]


@pytest.mark.parametrize("b, h, g, d, p, dtype, eight, length", MANY, ids=lambda x: str(x) if isinstance(x, int) else None)
def test_more_sequences_than_threads(b, h, g, d, p, dtype, eight, length):
    gen = torch.Generator(device="cuda").manual_seed(b)
    lens = [length(s) for s in range(b)]
    cache = filled(gen, b, h, g, d, p, dtype, eight, lens)
    q = torch.randn((b, h * g, d), generator=gen, device="cuda", dtype=dtype)
    for opt, first in (({}, None), ({"window": 20, "cap": 5.0}, torch.tensor([n // 3 for n in lens], dtype=torch.int32, device="cuda"))):
        out = nan_out(cache)
        cache.attend(q, ScoreMod(window=opt.get("window", 0), softcap=opt.get("cap", 0.0)), first_pos=first, out=out)
        check_attend(out, cache, q, opt, None, first)
    assert device_error_count() == 0


@pytest.mark.parametrize("b, h, g, n, length", [(300, 1, 4, 1, lambda s: s % 100), (900, 2, 2, 3, lambda s: 0 if s % 5 < 4 else s % 130)])
def test_few_rows_of_more_sequences_than_threads(b, h, g, n, length):
    d, gen = 64, torch.Generator(device="cuda").manual_seed(b)
    lens = [length(s) for s in range(b)]
    m = max(lens)
    q, k, v = rows(gen, b, h * g, n, d, BF16), rows(gen, b, h, m, d, BF16), rows(gen, b, h, m, d, BF16)
    ql, kl = torch.tensor([s % (n + 1) for s in range(b)], dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = make_cache(b, h, g, d, BF16)
    out = cache.attend_cross(q, k, v, ql, kl, out=torch.full_like(q, 7.0), workspace=cache.cross_workspace(n, m))
    s = q.double().view(b, h, g * n, d) @ k.double().mT / d ** 0.5
    s = s.masked_fill(torch.arange(m, device="cuda") >= kl[:, None, None, None], -torch.inf)
    want = (torch.nan_to_num(s.softmax(-1)) @ v.double()).view(b, h * g, n, d)
    inside = (torch.arange(n, device="cuda") < ql[:, None])[:, None, :, None].expand_as(out)
    assert bool((out[~inside] == 7.0).all())
    tol = tolerance(want, v.double().abs().max(), BF16, True)
    assert bool(((out.double() - want).abs() <= tol)[inside].all()) and device_error_count() == 0
