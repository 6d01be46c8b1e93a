"""The rotary and scored-attention operators from their definitions, in 64 bits, and the tolerances that follow from the kernels' arithmetic."""
import math

import torch


def rotate(x, pos, freq, amplitude, interleaved):
    """Rows x [..., d] at positions pos [...]; freq in radians per position (fp64)."""
    r, y = 2 * freq.numel(), x.double().clone()
    angle = pos.double()[..., None] * freq.to(x.device)
    cos, sin = angle.cos() * amplitude, angle.sin() * amplitude
    a, c = (y[..., 0:r:2].clone(), y[..., 1:r:2].clone()) if interleaved else (y[..., : r // 2].clone(), y[..., r // 2: r].clone())
    if interleaved:
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - c * sin, c * cos + a * sin
    else:
        y[..., : r // 2], y[..., r // 2: r] = a * cos - c * sin, c * cos + a * sin
    return y


def attend(q, k, v, t, p, seen, scale=0.0, cap=0.0, slopes=None):
    """softmax(x) v for one KV head: q [G, rows, d], k / v [n, d], t [rows], p [n], seen [rows, n]. Hidden keys are left out altogether."""
    q, v = q.double(), torch.where(seen.any(0)[:, None], v.double(), 0.0)
    k = torch.where(seen.any(0)[:, None], k.double(), 0.0)
    x = q @ k.T * (scale or 1 / math.sqrt(q.shape[-1]))
    if cap:
        x = cap * torch.tanh(x / cap)
    if slopes is not None:
        x = x - slopes.double()[:, None, None] * (t[:, None] - p[None, :]).abs().double()
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    w = torch.where(total > 0, w / total, 0.0)
    return w @ v


def prompt_seen(n, window=0, doc_start=None, prefix=0, device="cuda"):
    i, j = torch.arange(n, device=device)[:, None], torch.arange(n, device=device)[None]
    low = torch.zeros_like(i) if doc_start is None else doc_start[:n, None].long()
    if window:
        low = torch.maximum(low, i - window + 1)
    return (j >= low) & (j < torch.clamp(torch.maximum(i + 1, torch.full_like(i, prefix)), max=n))


def tolerance(ref, vmax, dtype, split):
    """How far an attention output may be from exact arithmetic. Scores, softmax and sums in fp32 leave each weight off by a few 1e-6
    (2e-5 of the largest |V|, as for he_attend). A kernel that rounds its weights to bf16 (`split` false) adds half a step of every
    weight, 2^-8 of it, so at most 2^-8 of the largest |V|; an output in bf16 adds half a step of itself."""
    tol = 2e-5 * vmax + torch.zeros_like(ref)
    if not split:
        tol = tol + 2.0 ** -8 * vmax
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * ref.abs()
    return tol
