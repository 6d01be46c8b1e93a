"""Attention around the cache at sizes and in kernels that short prompts do not reach."""
import pytest
import torch

import test_gpu_layer_ops
from paper_2412_16187_b200 import ScoreMod, binding
from test_gpu_layer_ops import BF16, F32, OPTIONS, SCORED, check_prompt, make_cache, prompt_case, rows

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


# Enough tiles for every SM: fp32 prompts then take tiles of 64 rows, whose copies are asynchronous; heads of every size that has a kernel of its own.
MANY = [(2, 4, 2, 64, F32, [700, 333], "heads"), (2, 2, 4, 128, F32, [690, 64], "tokens"), (1, 8, 2, 136, F32, [641], "heads"), (2, 4, 2, 192, F32, [700, 1], "tokens"),
        (2, 4, 2, 200, F32, [650, 127], "heads"), (1, 16, 1, 256, F32, [640], "tokens"), (2, 4, 2, 136, BF16, [700, 65], "tokens"), (1, 16, 1, 192, BF16, [641], "heads"),
        (2, 8, 1, 256, BF16, [640, 600], "tokens"), (2, 2, 4, 208, BF16, [700, 0], "heads"), (5, 4, 8, 40, F32, [60, 1, 0, 17, 33], "heads")]
FEW = [(1, 1, 2, 136, F32, [130], "heads"), (2, 1, 1, 192, F32, [65, 63], "tokens"), (1, 2, 1, 160, BF16, [200], "heads"), (1, 1, 3, 256, F32, [77], "heads")]


@pytest.mark.parametrize("opt", list(OPTIONS))
@pytest.mark.parametrize("shape", MANY + FEW, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}x{s[3]}-{'bf16' if s[4] == BF16 else 'fp32'}-{max(s[5])}")
def test_prompts_on_the_cuda_cores(shape, opt):
    o = OPTIONS[opt]
    q, k, v, plen, mod, kw, slopes = prompt_case(shape, o, seed=12)
    out = torch.full_like(q, 7.0)
    make_cache(*shape[:5]).attend_prompt(q, k, v, plen, mod=mod, out=out, **kw)
    check_prompt(out, q, k, v, shape[5], o, kw, slopes, shape[2], split=True)
    for s, n in enumerate(shape[5]):
        assert bool((out[s, :, n:] == 7.0).all())


@pytest.mark.parametrize("opt", ["plain", "all"])
def test_many_bf16_rows_without_tensor_cores(opt, monkeypatch):
    monkeypatch.setenv("HE_DISABLE_ATTEND_MMA", "1")
    test_prompts_on_the_cuda_cores((2, 4, 2, 96, BF16, [700, 311], "tokens"), opt)


@pytest.mark.parametrize("opt", list(SCORED))
@pytest.mark.parametrize("shape, fills", [((2, 2, 5, 64, F32), [150, 31]), ((1, 3, 8, 128, F32), [700]), ((200, 1, 8, 40, F32), [1 + s for s in range(200)]),
                                          ((1, 2, 2, 128, F32), [1300]), ((2, 2, 6, 256, F32), [90, 300]), ((160, 1, 1, 256, BF16), [70] * 160)],
                         ids=lambda x: "x".join(map(str, x[:4])) if isinstance(x, tuple) else str(max(x)))
def test_scored_attention_over_shared_memory_tiles(shape, fills, opt):
    test_gpu_layer_ops.test_attend_scored(shape, fills, opt)


@pytest.mark.parametrize("opt", list(SCORED))
@pytest.mark.parametrize("shape, fills", [((2, 2, 2, 128, BF16), [400, 63]), ((180, 1, 2, 64, BF16), [50] * 180), ((1, 1, 5, 128, BF16), [1500])],
                         ids=lambda x: "x".join(map(str, x[:4])) if isinstance(x, tuple) else str(max(x)))
def test_scored_attention_in_bf16_without_tensor_maps(shape, fills, opt, monkeypatch):
    monkeypatch.setenv("HE_DISABLE_ATTEND_MMA", "1")
    test_gpu_layer_ops.test_attend_scored(shape, fills, opt)
