"""Attention around the cache at sizes and in kernels that short prompts do not reach."""
import pytest
import torch

from paper_2412_16187_b200 import ScoreMod, binding
from test_gpu_layer_ops import BF16, make_cache, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d, group, mod", [(128, 4, None), (64, 1, ScoreMod(softcap=20.0)), (128, 3, ScoreMod(window=50))])
def test_most_of_the_work_lies_behind_the_prompts_ends(d, group, mod):
    """Short prompts in long rows: CTAs are handed one tile after another that has no tokens, and go on to those that do."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    b, h, n = 48, 2, 4000
    lens = [1 + (37 * s) % 90 for s in range(b)]
    lens[7], lens[20], lens[b - 1] = 0, 1500, 300
    q, k, v = rows(gen, b, h * group, n, d, BF16), rows(gen, b, h, n, d, BF16), rows(gen, b, h, n, d, BF16)
    out = torch.full_like(q, 7.0)
    make_cache(b, h, group, d, BF16).attend_prompt(q, k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), mod=mod, out=out)
    alone = make_cache(1, h, group, d, BF16)
    for s, m in enumerate(lens):
        assert bool((out[s, :, m:] == 7.0).all())
        if m:
            want = alone.attend_prompt(q[s:s + 1, :, :m], k[s:s + 1, :, :m], v[s:s + 1, :, :m], torch.tensor([m], dtype=torch.int32, device="cuda"), mod=mod)
            assert torch.equal(out[s, :, :m], want[0]), s
    assert binding.device_error_count() == 0
