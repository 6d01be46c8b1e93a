"""Caps far from the scores, beyond what the near form of the tanh can be written for, and hidden scores beside seen ones."""
import math

import pytest
import torch

from layer_reference import attend, prompt_seen, tolerance
from paper_2412_16187_b200 import ScoreMod
from test_gpu_layer_ops import BF16, F32, make_cache, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale, cap, size", [(1.0, 1e-7, 1e-5), (1.0, 2e-7, 3e-4), (4.0, 1e-8, 0.0), (1e3, 1e-9, 1e-8), (1.0, 1e-6, 1e-5), (1.0, 1e-5, 1e-4), (1e4, 1e-9, 1e-3)])
@pytest.mark.parametrize("dtype, d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_caps_far_below_the_products(scale, cap, size, dtype, d):
    """Every score lies within the cap, next to nothing: a row's output is the mean of the values that it sees."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    n = 300
    cache = make_cache(1, 1, 2, d, dtype)
    q, k = (rows(gen, 1, h, n, d, dtype).abs_().mul_(size) for h in (2, 1))
    v = rows(gen, 1, 1, n, d, dtype)
    out = cache.attend_prompt(q, k, v, torch.tensor([n], dtype=torch.int32, device="cuda"), mod=ScoreMod(scale=scale, softcap=cap))
    at = torch.arange(n, device="cuda")
    ref = attend(q[0], k[0, 0], v[0, 0], at, at, prompt_seen(n), scale=scale, cap=cap)
    # scores of at most 1e-5, whatever their relative error, leave weights within 2e-5 of one another
    tol = tolerance(ref, v.double().abs().max(), dtype, dtype == F32) + 2 * cap * v.double().abs().max()
    assert bool(((out[0].double() - ref).abs() <= tol).all()), float(((out[0].double() - ref).abs() - tol).max())


@pytest.mark.parametrize("dtype, d", [(BF16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("cap", [0.0, 2.0, 40.0])
@pytest.mark.parametrize("slopes", [False, True])
def test_no_bit_depends_on_a_key_that_is_hidden(dtype, d, cap, slopes):
    """Hidden keys that are NaN or infinite, next to seen ones in the block: the past ahead of each row's document, the window, the prompt's end."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, tokens = 301, 310
    cache = make_cache(1, 1, 2, d, dtype)
    q, k, v = rows(gen, 1, 2, tokens, d, dtype), rows(gen, 1, 1, tokens, d, dtype), rows(gen, 1, 1, tokens, d, dtype)
    plen = torch.tensor([n], dtype=torch.int32, device="cuda")
    doc = torch.full((1, tokens), 61, dtype=torch.int32, device="cuda")
    mod = ScoreMod(softcap=cap, slopes=torch.tensor([0.25, 0.01], device="cuda") if slopes else None)
    clean = cache.attend_prompt(q, k, v, plen, mod=mod, doc_start=doc, out=torch.zeros_like(q))
    for bad in (math.nan, math.inf):
        k[:, :, :61], k[:, :, n:] = bad, bad
        assert torch.equal(cache.attend_prompt(q, k, v, plen, mod=mod, doc_start=doc, out=torch.zeros_like(q)), clean), bad
