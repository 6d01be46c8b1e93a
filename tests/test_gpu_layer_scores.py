"""Attention of prompts and of rows over other keys with scores far from zero, against its definition in 64 bits."""
import pytest
import torch

from layer_reference import attend, tolerance
from paper_2412_16187_b200 import ScoreMod
from test_gpu_layer_ops import BF16, F32, make_cache

pytestmark = pytest.mark.gpu


# rows, keys, group: a prompt over itself (None); tiles over other keys, shares of the keys, several heads' rows in a tile, few rows
CALLS = {"prompt": (140, None, 2), "tiles": (140, 300, 2), "shares": (20, 700, 2), "one head": (70, 1500, 1), "few": (1, 700, 1)}


@pytest.mark.parametrize("cap", [0.0, 2.0 ** 26, 2.0 ** 34])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("call", list(CALLS))
def test_scores_of_any_size(call, dtype, d, cap):
    """One channel of q meets one of k, so that a score is exact up to one rounding: two are equal or far apart, and a row is the mean of the V rows whose score is the largest it
    sees. Scores of 2^10 to 2^48 in both signs, small ones ahead of them, a sequence each. With a cap all have the same magnitude, as beside its ends two would be closer than
    fp32 can tell."""
    n, m, g = CALLS[call]
    sizes = [x * 2.0 ** e for e in range(10, 44, 2) for x in (1.0, 1.3125, 1.75)]
    b, keys, gen = len(sizes), m or n, torch.Generator(device="cuda").manual_seed(d)
    q, k = torch.zeros((b, g, n, d), device="cuda", dtype=dtype), torch.zeros((b, 1, keys, d), device="cuda", dtype=dtype)
    v = torch.randn((b, 1, keys, d), generator=gen, device="cuda", dtype=dtype)
    k[..., 3] = 1.0 if cap else torch.randint(1, 16, (b, 1, keys), generator=gen, device="cuda").to(dtype)
    k[::3, :, ::2, 3] *= -1.0
    q[..., 3] = torch.tensor(sizes, device="cuda")[:, None, None] * torch.tensor([1.0, -1.0], device="cuda")[:g, None]
    q[..., 1::2, 3] *= 2.0 ** -30  # (rows beside far ones)
    cache, mod = make_cache(b, 1, g, d, dtype), ScoreMod(scale=1.0, softcap=cap)
    rows, lens = torch.full((b,), n, dtype=torch.int32, device="cuda"), torch.full((b,), keys, dtype=torch.int32, device="cuda")
    out = cache.attend_prompt(q, k, v, rows, mod=mod) if m is None else cache.attend_cross(q, k, v, rows, lens, mod=mod)
    at, t = torch.arange(keys, device="cuda"), torch.arange(n, device="cuda")
    seen = at <= t[:, None] if m is None else torch.ones((n, keys), dtype=torch.bool, device="cuda")
    for s in range(b):
        want = attend(q[s], k[s, 0], v[s, 0], t, at, seen, 1.0, cap)
        tol = tolerance(want, v[s, 0].double().abs().max(), dtype, dtype == F32)
        assert bool(((out[s].double() - want).abs() <= tol).all()), (sizes[s], float((out[s].double() - want).abs().max()))
