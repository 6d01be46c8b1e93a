"""One workspace of the attention over keys of another length for calls of many sizes."""
import random

import pytest
import torch

from paper_2412_16187_b200 import device_error_count
from test_gpu_layer_ops import BF16, F32, make_cache, rows

pytestmark = pytest.mark.gpu


# (B, H, G, d, dtype, rows and keys of the workspace, rows and keys of calls): the last, shorter chunks of a prompt, a new token, odd groups, other paths
CASES = [
    (1, 8, 4, 128, BF16, (512, 32768), [(512, 32768), (384, 32768), (300, 32768), (128, 32768), (114, 30000), (100, 32768), (64, 9000), (33, 32768), (2, 32768), (1, 32768), (512, 700)]),
    (1, 8, 4, 128, BF16, (1024, 32768), [(1024, 32768), (512, 32768), (130, 20000), (1, 32768), (1, 100)]), (3, 2, 7, 64, BF16, (300, 5000), [(300, 5000), (150, 5000), (32, 4000), (1, 5000)]),
    (2, 2, 2, 64, F32, (200, 3000), [(200, 3000), (64, 3000), (17, 2000), (16, 3000), (1, 3000)]), (1, 1, 3, 256, BF16, (100, 4000), [(100, 4000), (40, 4000), (3, 1000)]),
]


@pytest.mark.parametrize("b, h, g, d, dtype, most, calls", CASES, ids=lambda x: str(x) if isinstance(x, (int, tuple)) else None)
def test_a_workspace_serves_every_shorter_call(b, h, g, d, dtype, most, calls):
    """With the same results, bit for bit, as a workspace of the call's own sizes, and as a call that makes its own."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    q, k, v = rows(gen, b, h * g, most[0], d, dtype), rows(gen, b, h, most[1], d, dtype), rows(gen, b, h, most[1], d, dtype)
    cache = make_cache(b, h, g, d, dtype)
    ws = cache.cross_workspace(*most)
    assert ws.numel() > 0
    ws.fill_(255)
    for n, m in calls:
        part, keys, values = q[:, :, :n], k[:, :, :m], v[:, :, :m]
        ql, kl = (torch.full((b,), x, dtype=torch.int32, device="cuda") for x in (n, m))
        for pos in (None, kl - ql):
            got, own = (cache.attend_cross(part, keys, values, ql, kl, q_pos=pos, workspace=x) for x in (ws, cache.cross_workspace(n, m)))
            assert torch.equal(got, own) and torch.equal(got, cache.attend_cross(part, keys, values, ql, kl, q_pos=pos)) and bool(torch.isfinite(got).all())
    assert device_error_count() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_shorter_call_is_refused(dtype):
    rng = random.Random(4)
    for _ in range(6):
        b, h, g, d = rng.choice((1, 1, 2, 5)), rng.choice((1, 2, 8)), rng.choice((1, 2, 3, 8)), rng.choice((16, 64, 128))
        n, m = rng.randint(1, 600), rng.randint(1, 20000)
        cache = make_cache(b, h, g, d, dtype)
        ws = cache.cross_workspace(n, m)
        q, k = torch.zeros((b, h * g, n, d), dtype=dtype, device="cuda"), torch.zeros((b, h, m, d), dtype=dtype, device="cuda")
        lens = torch.zeros((b,), dtype=torch.int32, device="cuda")  # (nothing to compute: what counts is that the call is taken)
        for _ in range(30):
            a, c = rng.randint(1, n), rng.randint(1, m)
            cache.attend_cross(q[:, :, :a], k[:, :, :c], k[:, :, :c], lens, lens, out=q[:, :, :a].clone(), workspace=ws)
