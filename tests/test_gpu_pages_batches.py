"""Attention over pages for padded batches: sequences that see nothing beside others."""
import pytest
import torch

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
