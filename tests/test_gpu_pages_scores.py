"""Attention over 8-bit pages with scores far from zero, against its definition in 64 bits."""
import pytest
import torch

from layer_reference import tolerance
from paper_2412_16187_b200 import ScoreMod
from test_gpu_layer_ops import BF16, F32
from test_gpu_pages import filled, check_attend, paged

pytestmark = pytest.mark.gpu

SHAPES = [(2, 4, 128, 64, BF16), (1, 8, 128, 16, BF16), (2, 3, 64, 32, BF16), (1, 4, 128, 128, F32), (1, 5, 64, 16, F32)]  # KV heads, group, d, page, dtype
NAMES = ["x".join(map(str, s[:4])) + ("-bf16" if s[4] == BF16 else "-fp32") for s in SHAPES]


@pytest.mark.parametrize("cap", [0.0, 2.0 ** 26])
@pytest.mark.parametrize("h, g, d, p, dtype", SHAPES, ids=NAMES)
def test_scores_of_any_size(h, g, d, p, dtype, cap):
    """One channel of q meets one of K, so that every score is exact up to one rounding: two are equal or far apart, and a row is the mean of the V rows whose score is the
    largest. Scores of 2^17 to 2^32 in both signs (a head's q has its own), a sequence each. With a cap all have the same magnitude: beside its ends two of them would be
    closer than fp32 can tell."""
    sizes = [m * 2.0 ** e for e in range(17, 29) for m in (1.0, 1.3125, 1.75)]
    b, n = len(sizes), 300
    gen = torch.Generator(device="cuda").manual_seed(d + p)
    cache = paged(gen, b, h, g, d, p, dtype, True, n)
    k, v = torch.zeros((b, h, n, d), device="cuda", dtype=dtype), torch.randn((b, h, n, d), generator=gen, device="cuda", dtype=dtype)
    k[..., 3] = 1.0 if cap else torch.randint(1, 16, (b, h, n), generator=gen, device="cuda").to(dtype)  # (e4m3 has four bits)
    k[::3, :, ::2, 3] *= -1.0
    q = torch.zeros((b, h * g, d), device="cuda", dtype=dtype)
    q[..., 3] = torch.tensor(sizes, device="cuda")[:, None] * torch.tensor([1.0, -1.0] * (h * g), device="cuda")[: h * g]
    cache.length += n
    cache.append(k, v)
    got = cache.attend(q, ScoreMod(scale=1.0, softcap=cap)).double()
    assert bool(torch.isfinite(got).all())
    check_attend(got, cache, q, {"scale": 1.0, "cap": cap}, None, None)


@pytest.mark.parametrize("h, g, d, p, dtype", SHAPES, ids=NAMES)
def test_a_steep_bias(h, g, d, p, dtype):
    """Biases of up to 2^32 by distance: what lies far behind weighs nothing, and is no NaN either where a share of the work has nothing else."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    lens = [3000, 700, 33]
    cache = filled(gen, len(lens), h, g, d, p, dtype, True, lens)
    q = torch.randn((len(lens), h * g, d), generator=gen, device="cuda", dtype=dtype)
    for e in (8, 14, 15, 16, 21):
        slopes = torch.exp2(e - torch.arange(h * g, device="cuda") * 0.3)
        got = cache.attend(q, ScoreMod(slopes=slopes))
        assert bool(torch.isfinite(got).all())
        check_attend(got, cache, q, {}, slopes, None)


@pytest.mark.parametrize("h, g, d, p, dtype", SHAPES, ids=NAMES)
def test_a_scale_and_a_query_whose_product_leaves_fp32(h, g, d, p, dtype):
    """A page's scale comes from a row that is hidden; the visible rows' codes are zeros, and so are their scores, however large the query is: the mean of V."""
    gen = torch.Generator(device="cuda").manual_seed(p)
    n = 3 * p
    cache = paged(gen, 2, h, g, d, p, dtype, True, n)
    k, v = torch.zeros((2, h, n, d), device="cuda", dtype=dtype), torch.randn((2, h, n, d), generator=gen, device="cuda", dtype=dtype)
    k[:, :, p, 1], k[:, :, p + 1:, 2] = 2.0 ** 70, 1.0
    q = torch.full((2, h * g, d), 2.0 ** 100, device="cuda", dtype=dtype)
    cache.length += n
    cache.append(k, v)
    first = torch.full((2,), p + 1, dtype=torch.int32, device="cuda")
    cache.length.fill_(2 * p)  # (the scale of the third page is that of its own rows)
    v = cache.read(2 * p)[1][:, :, p + 1:].double()
    for cap in (0.0, 30.0):
        got = cache.attend(q, ScoreMod(softcap=cap), first_pos=first).double().view(2, h, g, d)
        want = v.mean(2)[:, :, None].expand_as(got)
        assert bool(((got - want).abs() <= tolerance(want, v.abs().max(), F32, True)).all())


@pytest.mark.parametrize("h, g, d, p, dtype", SHAPES, ids=NAMES)
def test_queries_with_an_infinity(h, g, d, p, dtype):
    """Scores of -inf alone give zeros, of +inf NaN; a cap makes both finite, here all equal: the mean of V."""
    gen = torch.Generator(device="cuda").manual_seed(d * p)
    n = 2 * p + 5
    cache = paged(gen, 2, h, g, d, p, dtype, True, n)
    k, v = (torch.randn((2, h, n, d), generator=gen, device="cuda", dtype=dtype) for _ in "kv")
    k[..., 3] = k[..., 3].abs() + 1.0
    q = torch.randn((2, h * g, d), generator=gen, device="cuda", dtype=dtype)
    q[:, 0::2, 3], q[:, 1::2, 3] = torch.inf, -torch.inf
    cache.length += n
    cache.append(k, v)
    got = cache.attend(q)
    assert bool(torch.isnan(got[:, 0::2]).all()) and not got[:, 1::2].any()
    got = cache.attend(q, ScoreMod(softcap=20.0)).double().view(2, h, g, d)
    values = cache.read(n)[1].double()
    want = values.mean(2)[:, :, None].expand_as(got)
    assert bool(((got - want).abs() <= tolerance(want, values.abs().max(), F32, True)).all())
