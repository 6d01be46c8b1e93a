"""Caps far below the products of q and k, whose ratio to the scale is beyond what the near form of the tanh can be written for."""
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
