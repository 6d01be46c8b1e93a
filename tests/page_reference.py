"""The paged cache from its definition, with torch on the pages' own bits: every code and scale that an append leaves is decided by it."""
import torch

E4M3 = torch.float8_e4m3fn


def scale_of(top):
    """The least power of two s >= 2^-100 with top <= 448 s, found by trying."""
    s = torch.full_like(top, 2.0 ** -100)
    for e in range(-99, 128):
        s = torch.where(top > 448 * s.double(), torch.full_like(s, 2.0 ** e), s)
    return s


def codes_of(x, s):
    """e4m3 of x / s to nearest even, NaN for what is not finite. (x / s is exact: a power of two, and in fp32 no smaller than 2^-120 of the page's largest counts.)"""
    y = (x.double() / s.double()).float()
    return torch.where(torch.isfinite(x), y, torch.nan).to(E4M3)


def append(model, rows, new_len):
    """model: dict with k_pages, v_pages [n_pages, H, P, d], k_scale, v_scale (8 bits) or None, page_table, length; rows = (k, v) [B, H, N, d], keys rotated already."""
    p = model["k_pages"].shape[2]
    n_pages, cap = model["k_pages"].shape[0], model["page_table"].shape[1] * p
    for s in range(rows[0].shape[0]):
        n = rows[0].shape[2] if new_len is None else min(max(int(new_len[s]), 0), rows[0].shape[2])
        held = max(int(model["length"][s]), 0)
        first = held - n
        for at in range(max(first, 0) // p, (min(held, cap) + p - 1) // p):
            page = int(model["page_table"][s, at])
            lo, hi = max(first, 0, at * p), min(held, cap, at * p + p)
            if lo >= hi or not 0 <= page < n_pages:
                continue
            for x, r in zip("kv", rows):
                pages, y = model[x + "_pages"], r[s, :, lo - first: hi - first]
                if pages.dtype != E4M3:
                    pages[page, :, lo - at * p: hi - at * p] = y
                    continue
                top = torch.where(torch.isfinite(y), y.double().abs(), 0.0).amax((1, 2))
                scale = scale_of(top).float()
                if lo > at * p:
                    old = model[x + "_scale"][page]
                    scale = torch.maximum(scale, old)
                    was = pages[page, :, : lo - at * p].float()
                    moved = (was.double() * (old / scale).double()[:, None, None]).float().to(E4M3)
                    pages.view(torch.uint8)[page, :, : lo - at * p] = moved.view(torch.uint8)
                model[x + "_scale"][page] = scale
                pages.view(torch.uint8)[page, :, lo - at * p: hi - at * p] = codes_of(y.float(), scale[:, None, None]).view(torch.uint8)


def values(model, x, s, n):
    """The first n rows of sequence s in 64 bits, [H, n, d]; zeros for pages that are not there."""
    pages, p = model[x + "_pages"], model["k_pages"].shape[2]
    ids = model["page_table"][s, : (n + p - 1) // p].long()
    there = (ids >= 0) & (ids < pages.shape[0])
    ids = ids.clamp(0, pages.shape[0] - 1)
    rows = pages.view(torch.uint8)[ids].view(E4M3).double() if pages.dtype == E4M3 else pages[ids].double()
    if pages.dtype == E4M3:
        rows = rows * model[x + "_scale"][ids].double()[:, :, None, None]
    rows = torch.where(there[:, None, None, None], rows, 0.0)
    return rows.transpose(0, 1).flatten(1, 2)[:, :n]
