"""How far attention outputs are from exact arithmetic, row by row, against what the roundings of the kernels can leave.

Bounds. A weight w_j whose relative error is e_j moves channel c by e_j w_j v_jc. The errors of different keys have nothing to do with the values, so over the d
channels of a row the squares add up and the mixed terms cancel to within 4 / sqrt(d) of the squares (four standard deviations): the root mean square over the
channels stays below sqrt(1 + 4 / sqrt(d)) times that of
    sqrt( sum_j (e_j w_j v_jc)^2 + (r o_c)^2 ),
with e_j the most that a weight may be off, and r what the output itself is rounded by.
  In fp32: exp2 is within 2 ulp, 2^-22; a score's sum of products S_j = scale * sum |q_c k_c| is rounded along the way, to within 2^-22 S_j, as is what the cap and
  the bias add to it. So e_j = 2^-22 (1 + S_j + |bias_j| + cap); r = 2^-22 for the last sums and the division; the sum over n keys in some order adds
  roundings of 2^-23 of its parts, whose squares come to n sum_j (w_j v_jc)^2 at most where the parts have either sign.
  Weights rounded to bf16: e_j = 2^-8. Outputs rounded to bf16: r = 2^-8.
A key too many or too few among n moves a row by about 1 / n of the values, ten times the bound in bf16 at 300 keys."""
import math

import pytest
import torch

from layer_reference import prompt_seen
from paper_2412_16187_b200 import ScoreMod
from test_gpu_layer_ops import BF16, F32, OPTIONS, fill_cache, make_cache, prompt_case

pytestmark = pytest.mark.gpu


def exact(q, k, v, t, p, seen, scale, cap, slopes):
    """Outputs and the bound's sums for one KV head: q [G, rows, d], k / v [n, d], t [rows], p [n], seen [rows, n]."""
    d = q.shape[-1]
    q, k, v = q.double(), k.double(), v.double()
    scale = scale or 1 / math.sqrt(d)
    x, size = q @ k.T * scale, q.abs() @ k.abs().T * scale
    if cap:
        x, size = cap * torch.tanh(x / cap), size + cap
    if slopes is not None:
        bias = slopes.double()[:, None, None] * (t[:, None] - p[None]).abs().double()
        x, size = x - bias, size + bias
    x = x.masked_fill(~seen, -math.inf)
    w = torch.softmax(x, -1).nan_to_num(0.0)
    keys = seen.sum(-1)[:, None].double()
    return w @ v, ((2.0 ** -22 * (1 + size) * w) ** 2) @ v ** 2 + 2.0 ** -46 * keys * (w ** 2 @ v ** 2), w ** 2 @ v ** 2


def check(got, o, fine, squares, bf16_weights, bf16_out):
    d = o.shape[-1]
    bound = fine + (2.0 ** -22 * o) ** 2
    if bf16_weights:
        bound = bound + 2.0 ** -16 * squares
    if bf16_out:
        bound = bound + (2.0 ** -8 * o) ** 2
    rms, most = ((got.double() - o) ** 2).mean(-1).sqrt(), ((1 + 4 / math.sqrt(d)) * bound.mean(-1)).sqrt()
    assert bool((rms <= most).all()), float((rms / most.clamp(min=1e-300)).max())


SHAPES = [(1, 2, 4, 128, BF16, [700], "heads"), (2, 4, 1, 64, BF16, [300, 513], "tokens"), (1, 1, 2, 96, BF16, [1100], "heads"), (1, 4, 2, 256, BF16, [300], "heads"),
          (2, 4, 2, 64, F32, [700, 100], "heads"), (1, 1, 2, 128, F32, [300], "heads"), (1, 8, 2, 200, F32, [641], "tokens"), (1, 1, 1, 136, F32, [200], "heads")]


@pytest.mark.parametrize("opt", list(OPTIONS))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}x{s[3]}-{'bf16' if s[4] == BF16 else 'fp32'}-{max(s[5])}")
def test_every_row_of_a_prompt(shape, opt):
    b, h, g, d, dtype, lens, _ = shape
    o = OPTIONS[opt]
    q, k, v, plen, mod, kw, slopes = prompt_case(shape, o, seed=31)
    out = make_cache(b, h, g, d, dtype).attend_prompt(q, k, v, plen, mod=mod, **kw)
    for s, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        seen = prompt_seen(n, o.get("window", 0), None if kw["doc_start"] is None else kw["doc_start"][s], 0 if kw["prefix_len"] is None else int(kw["prefix_len"][s]))
        for u in range(h):
            sl = slice(u * g, u * g + g)
            parts = exact(q[s, sl, :n], k[s, u, :n], v[s, u, :n], at, at, seen, o.get("scale", 0.0), o.get("cap", 0.0), None if slopes is None else slopes[sl])
            check(out[s, sl, :n], *parts, dtype == BF16 and d <= 128, dtype == BF16)


@pytest.mark.parametrize("slots", [3, 20, 32, 90, 700])
@pytest.mark.parametrize("b, h, g, d, dtype", [(160, 1, 4, 128, BF16), (160, 1, 8, 128, BF16), (4, 2, 4, 64, BF16), (4, 2, 7, 64, BF16), (160, 1, 3, 96, BF16), (2, 2, 1, 40, BF16),
                                               (8, 2, 2, 256, BF16), (8, 2, 4, 128, F32), (160, 1, 8, 64, F32)])
@pytest.mark.parametrize("opt", [{}, {"cap": 3.0}, {"slopes": True, "window": 2000}])
def test_weights_over_the_cache_keep_their_24_bits(slots, b, h, g, d, dtype, opt):
    """Two bf16 terms of a weight would leave up to 2^-17 of it, about twice the bound over up to 90 slots."""
    gen = torch.Generator(device="cuda").manual_seed(slots + d)
    cache = fill_cache(gen, (b, h, g, d, dtype), [slots] * b)
    q = (0.1 * torch.randn((b, h * g, d), generator=gen, device="cuda")).to(dtype)  # scores of about 0.1: weights of about the same size
    slopes = torch.full((h * g,), 0.001, device="cuda") if "slopes" in opt else None
    got = cache.attend_scored(q, ScoreMod(softcap=opt.get("cap", 0.0), window=opt.get("window", 0), slopes=slopes))
    for s in range(min(b, 4)):
        for u in range(h):
            sl, p = slice(u * g, u * g + g), cache.pos[s, u, :slots].long()
            now = cache.next_pos[s, u].long().reshape(1) - 1
            seen = (p > now - opt["window"])[None] if "window" in opt else torch.ones((1, slots), dtype=torch.bool, device="cuda")
            parts = exact(q[s, sl][:, None], cache.k_cache[s, u, :slots], cache.v_cache[s, u, :slots], now, p, seen, 0.0, opt.get("cap", 0.0), None if slopes is None else slopes[sl])
            # over all heads of a unit together: a row of few slots has few roundings
            o, fine, squares = (x[:, 0].reshape(-1) for x in parts)
            check(got[s, sl].reshape(-1), o, fine, squares, False, False)
