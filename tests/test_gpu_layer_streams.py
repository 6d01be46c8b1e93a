"""Outputs that a call makes for itself belong to the stream that it is enqueued on."""
import pytest
import torch

from paper_2412_16187_b200 import Rotary
from test_gpu_layer_ops import BF16, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["rotate_prompt", "rotate_step", "attend_prompt", "attend_scored", "attend", "decode_step"])
def test_an_output_of_another_stream_takes_no_memory_that_is_still_read(call):
    b, h, g, d, n = 64, 8, 2, 64, 64
    cache, other, rot = make_cache(b, h, g, d, BF16), torch.cuda.Stream(), Rotary(d)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k = (torch.randn((b, x, n, d), generator=gen, device="cuda").to(BF16) for x in (h * g, h))
    plen = torch.full((b,), n, dtype=torch.int32, device="cuda")
    one_q, one_k = q[:, :, 0].contiguous(), k[:, :, 0].contiguous()
    calls = {"rotate_prompt": lambda: cache.rotate_prompt(rot, q, None, stream=other)[0], "rotate_step": lambda: cache.rotate_step(rot, one_q, None, stream=other)[0],
             "attend_prompt": lambda: cache.attend_prompt(q, k, k, plen, stream=other), "attend_scored": lambda: cache.attend_scored(one_q, stream=other), "attend": lambda: cache.attend(one_q, stream=other),
             "decode_step": lambda: cache.decode_step(one_q, one_k, one_k, stream=other)}
    cache.fill.zero_()
    for _ in range(3):
        want = calls[call]().clone()  # (warm: no allocation or loading of code below)
    torch.cuda.synchronize()
    del want
    out = calls[call]()
    shape, dtype = out.shape, out.dtype
    torch.cuda.synchronize()
    del out
    torch.cuda.empty_cache()
    marked = torch.full(shape, 50, dtype=dtype, device="cuda")
    kept = torch.zeros_like(marked)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)  # about ten milliseconds
    kept.copy_(marked)
    del marked  # its memory is free for whatever this stream does next, and for this stream alone
    out = calls[call]()
    torch.cuda.synchronize()
    assert bool((kept == 50).all())
    assert out.shape == shape and not bool((out == 50).all())
