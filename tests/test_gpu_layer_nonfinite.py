"""Scores that are not numbers in the attention of a new token over the cache: they reach the rows that see them and nobody else."""
import math

import pytest
import torch

from paper_2412_16187_b200 import ScoreMod
from test_gpu_layer_ops import BF16, F32, fill_cache

pytestmark = pytest.mark.gpu

# one CTA a unit and clusters, with and without the third terms in empty rows, tensor maps and shared-memory tiles
CACHES = [((160, 1, 4, 128, BF16), 70), ((1, 2, 4, 128, BF16), 900), ((2, 1, 8, 64, BF16), 700), ((1, 1, 1, 80, BF16), 300), ((1, 1, 3, 256, BF16), 200),
          ((200, 1, 2, 64, F32), 40), ((1, 2, 4, 128, F32), 700), ((1, 1, 8, 64, F32), 130)]
NAMES = [f"{'x'.join(map(str, s[:4]))}-{'bf16' if s[4] == BF16 else 'fp32'}-{n}" for s, n in CACHES]


def filled(shape, slots, seed=17):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cache = fill_cache(gen, shape, [slots] * shape[0])
    q = torch.randn((shape[0], shape[1] * shape[2], shape[3]), generator=gen, device="cuda", dtype=shape[4])
    return cache, q


@pytest.mark.parametrize("shape, slots", CACHES, ids=NAMES)
@pytest.mark.parametrize("call", ["scored", "capped", "attend"])
def test_a_query_that_is_not_a_number_gives_none(shape, slots, call):
    cache, q = filled(shape, slots)
    run = {"scored": lambda: cache.attend_scored(q), "capped": lambda: cache.attend_scored(q, ScoreMod(softcap=9.0)), "attend": lambda: cache.attend(q)}[call]
    clean = run()
    assert bool(torch.isfinite(clean).all())
    last = shape[1] * shape[2] - 1
    q[0, last, 5] = math.nan
    got = run()
    assert bool(torch.isnan(got[0, last]).all())
    others = torch.ones(got.shape[:2], dtype=torch.bool, device="cuda")
    others[0, last] = False
    assert torch.equal(got[others], clean[others])


@pytest.mark.parametrize("shape, slots", CACHES, ids=NAMES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("call", ["scored", "window", "attend"])
def test_a_visible_key_that_is_not_finite_reaches_its_unit(shape, slots, bad, call):
    """A NaN, or an infinity that makes a score +inf: the weights are inf - inf. Hidden by the window it touches nobody."""
    cache, q = filled(shape, slots)
    g, u = shape[2], shape[1] - 1
    q[0, u * g:, 3] = 1.0
    mod = ScoreMod(window=slots) if call == "window" else None
    run = (lambda: cache.attend(q)) if call == "attend" else (lambda: cache.attend_scored(q, mod))
    clean = run()
    age = cache.next_pos[0, u] - 1 - cache.pos[0, u, :slots]
    if call == "window":
        oldest = int(age.argmax())
        assert int(age[oldest]) >= slots  # hidden
        cache.k_cache[0, u, oldest, 3] = bad
        assert torch.equal(run(), clean)
    cache.k_cache[0, u, int(age.argmin()), 3] = bad
    got = run()
    assert bool(torch.isnan(got[0, u * g:]).all())
    others = torch.ones(got.shape[:2], dtype=torch.bool, device="cuda")
    others[0, u * g:] = False
    assert torch.equal(got[others], clean[others]) and bool(torch.isfinite(clean).all())


@pytest.mark.parametrize("shape, slots", CACHES, ids=NAMES)
@pytest.mark.parametrize("call", ["scored", "attend"])
def test_scores_of_minus_infinity_have_no_weight(shape, slots, call):
    """The first 33 slots (fewer than all) of a unit: whoever walks over them first sees nothing else for a while."""
    cache, q = filled(shape, slots)
    g, u, first = shape[2], shape[1] - 1, min(33, slots - 3)
    q[0, u * g:, 3] = 1.0
    run = cache.attend if call == "attend" else cache.attend_scored
    cache.k_cache[0, u, :first, 3] = -math.inf
    got = run(q)[0, u * g:].double()
    k, v = cache.k_cache[0, u, first:slots].double(), cache.v_cache[0, u, first:slots].double()
    want = torch.softmax(q[0, u * g:].double() @ k.T / math.sqrt(shape[3]), -1) @ v
    # scores, weights and sums in fp32: a few 1e-6 of the largest |V|
    assert bool(((got - want).abs() <= 2e-5 * float(cache.v_cache[0, u, :slots].double().abs().max())).all())


def test_a_unit_whose_scores_are_all_minus_infinity_gives_zeros():
    for shape, slots in CACHES:
        cache, q = filled(shape, slots)
        g, u = shape[2], shape[1] - 1
        q[0, u * g:, 3] = 1.0
        cache.k_cache[0, u, :slots, 3] = -math.inf
        assert not cache.attend(q)[0, u * g:].any() and not cache.attend_scored(q)[0, u * g:].any()
