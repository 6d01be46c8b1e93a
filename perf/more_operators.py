"""What is measured of the paged cache of the full history and of attention over keys of another length.

A case is a flat dict:
  op        "append": keys, rotated by their positions on the way, and values of new tokens into a paged cache
            "attend": attention of one new token per sequence over its pages
            "read": rows of the pages as plain keys and values
            "cross": attention of rows over keys of another length (a chunk of a prompt over all that came before it, or encoder states)
  batch, kv_heads, group, dim, dtype      shape of a layer (bf16 or f32)
  lo, hi    tokens that a cache holds, or keys, uniform in that range, a sequence each
paged:  store ("same": pages in the dtype, "e4m3": 8 bits with a scale for each page and head), page (tokens of a page)
append: new_lo, new_hi (the call's tokens of a sequence, the last of those that it holds), rot ("none", "half" or "inter" pairs), layout
attention: cap (tanh cap of the scores, 0: none), slopes (distance bias), window (0: none), docs (thousandths of the positions that belong to earlier
          documents, single tokens only)
read:   skip (thousandths of a sequence that are left out ahead of the rows)
cross:  new_lo, new_hi (rows of a sequence), causal (the rows are the last of the keys' positions, each sees what is not behind it), layout
layout "heads": [batch, heads, tokens, dim] in memory, "tokens": [batch, tokens, heads, dim], as a projection leaves them
"""
import math

import torch

own = False
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------------------------ cases
def _shape(name, op, batch, kv_heads, group, dim, dtype, lo, hi):
    return {"name": name, "op": op, "batch": batch, "kv_heads": kv_heads, "group": group, "dim": dim, "dtype": dtype, "lo": lo, "hi": hi}


def _append(name, *shape, store, page, new_lo, new_hi, rot="half", layout="heads"):
    return {**_shape(name, "append", *shape), "store": store, "page": page, "new_lo": new_lo, "new_hi": new_hi, "rot": rot, "layout": layout}


def _attend(name, *shape, store, page, cap=0.0, slopes=False, window=0, docs=0):
    return {**_shape(name, "attend", *shape), "store": store, "page": page, "cap": cap, "slopes": slopes, "window": window, "docs": docs}


def _read(name, *shape, store, page, skip=0):
    return {**_shape(name, "read", *shape), "store": store, "page": page, "skip": skip}


def _cross(name, *shape, new_lo, new_hi, causal, cap=0.0, slopes=False, window=0, layout="heads"):
    return {**_shape(name, "cross", *shape), "new_lo": new_lo, "new_hi": new_hi, "causal": causal, "cap": cap, "slopes": slopes, "window": window,
            "layout": layout}


def listed():
    return [
        # --- keys and values into the pages
        # one token of the tiny configuration: nothing but the latency of a call
        _append("append step tiny fp32", 1, 4, 1, 64, "f32", 65, 65, store="same", page=16, new_lo=1, new_hi=1),
        # one token of each of the throughput batch's 64 sequences, somewhere in a page of 8-bit rows
        _append("append step x64, 8 bit", 64, 8, 4, 128, "bf16", 512, 4096, store="e4m3", page=64, new_lo=1, new_hi=1),
        # ragged prompts straight from the projection, behind what their sequences hold already
        _append("append prompts x16, 8 bit", 16, 8, 4, 128, "bf16", 4500, 8192, store="e4m3", page=64, new_lo=1024, new_hi=4400, layout="tokens"),
        # --- attention of a new token over the pages
        # the tiny configuration in fp32: latency
        _attend("pages tiny fp32, bias", 1, 4, 1, 64, "f32", 128, 128, store="same", page=16, slopes=True),
        # the throughput batch, 8 bits, capped scores
        _attend("pages ragged x64, 8 bit, cap", 64, 8, 4, 128, "bf16", 512, 4096, store="e4m3", page=64, cap=30.0),
        # the long-context layer at batch 1, 8 bits
        _attend("pages long, 8 bit", 1, 8, 4, 128, "bf16", 32768, 32768, store="e4m3", page=128),
        # ragged sequences in bf16, bias by distance, the earlier documents hidden
        _attend("pages x16 bf16, bias + doc", 16, 8, 4, 128, "bf16", 1024, 8192, store="same", page=32, slopes=True, docs=250),
        # --- rows back out of the pages, as the compression and the attention loss take them
        _read("read one short, fp32", 1, 4, 1, 64, "f32", 130, 130, store="same", page=16),
        _read("read ragged x16, 8 bit", 16, 8, 4, 128, "bf16", 1024, 8192, store="e4m3", page=64),
        # --- rows over keys of another length
        # one decoder token of each of 8 sequences over its encoder's states: the latency of a call with few rows
        _cross("cross step x8, d64", 8, 16, 1, 64, "bf16", 700, 1500, new_lo=1, new_hi=1, causal=False),
        # ragged decoder prompts over encoder states, rows as the projection leaves them
        _cross("cross ragged x8, cap", 8, 16, 1, 64, "bf16", 700, 1500, new_lo=100, new_hi=448, causal=False, cap=50.0, layout="tokens"),
        # a chunk of a long prompt over all that came before it
        _cross("chunk of 512 in 32768", 1, 8, 4, 128, "bf16", 32768, 32768, new_lo=512, new_hi=512, causal=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Shapes of a transformer layer (1 to 32 KV heads, groups of 1 to 8, heads of 64 to 128), 1 to 64 sequences of up to 32768 tokens, every page size and
    store, and every combination of the options that a call takes."""
    while True:
        op = rng.choice(("append", "append", "attend", "attend", "attend", "read", "cross", "cross"))
        dtype = "f32" if rng.random() < 0.15 else "bf16"
        shape = (_log(rng, 1, 64), rng.choice((1, 2, 4, 8, 8, 32)), rng.choice((1, 2, 4, 4, 4, 7, 8)), rng.choice((64, 80, 96, 128, 128, 128)), dtype)
        batch, heads, group, dim, _ = shape
        hi = _log(rng, 8, 32768)
        lo = rng.randint(max(1, hi // 8), hi)
        e = 4 if dtype == "f32" else 2
        paged = {"store": rng.choice(("same", "e4m3", "e4m3")), "page": rng.choice((16, 32, 64, 128))}
        scores = {"cap": rng.choice((0.0, 0.0, 20.0, 50.0)), "slopes": rng.random() < 0.3, "window": rng.choice((0, 0, 0, _log(rng, 16, 8192)))}
        layout = rng.choice(("heads", "tokens"))
        if op == "append":
            new_hi = rng.choice((1, rng.randint(1, lo), rng.randint(1, lo)))
            c = _append("", *shape, lo, hi, **paged, new_lo=rng.randint(max(1, new_hi // 4), new_hi), new_hi=new_hi, rot=rng.choice(("none", "half", "half", "inter")),
                        layout=layout)
            if batch * heads * dim * hi * e > 16 * 8 * 128 * 8192 * 2 or batch * heads * dim * new_hi * e > 16 * 8 * 128 * 4400 * 2:
                continue
        elif op == "attend":
            c = _attend("", *shape, lo, hi, **paged, **scores, docs=rng.choice((0, 0, rng.randint(1, 900))))
            if batch * heads * dim * hi * (e if paged["store"] == "same" else 1) > 16 * 8 * 128 * 8192 * 2:
                continue
        elif op == "read":
            c = _read("", *shape, lo, hi, **paged, skip=rng.choice((0, rng.randint(0, 900))))
            if batch * heads * dim * hi * e > 16 * 8 * 128 * 8192 * 2:
                continue
        else:
            causal = rng.random() < 0.5
            if not causal:
                scores.update(slopes=False, window=0)
            new_hi = _log(rng, 1, min(lo, 4096) if causal else 4096)
            c = _cross("", *shape, lo, hi, new_lo=rng.randint(max(1, new_hi // 4), new_hi), new_hi=new_hi, causal=causal, **scores, layout=layout)
            if batch * heads * group * new_hi * hi > 512 * 32 * 32768 // (1 if dtype == "bf16" else 16) or batch * heads * dim * hi * e > 16 * 8 * 128 * 8192 * 2:
                continue
        del c["name"]
        return c


def _lengths(case):
    """Tokens that the sequences hold (keys), and how many of them are new (rows). Part of the case: two seeds of it differ in values only."""
    g = torch.Generator().manual_seed(case["lo"] * 1_000_003 + case["hi"])
    held = torch.randint(case["lo"], case["hi"] + 1, (case["batch"],), generator=g)
    new = torch.randint(case.get("new_lo", 1), case.get("new_hi", 1) + 1, (case["batch"],), generator=g)
    return held, new


def _frequencies(case):
    return 500000.0 ** (-2.0 * torch.arange(case["dim"] // 2, dtype=torch.float64) / case["dim"])


# ----------------------------------------------------------------------------------------------------------------- inputs
class _Maker:
    """Rows with the outlier channels that keys of trained layers show, from one seed."""

    def __init__(self, case, seed):
        self.case, self.g = case, torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=_DT[self.case["dtype"]])

    def rows(self, heads, tokens):
        """[batch, heads, tokens, dim], in memory as the case lays its rows out."""
        b, d = self.case["batch"], self.case["dim"]
        if self.case.get("layout") == "tokens":
            return self.normal(b, tokens, heads, d).transpose(1, 2)
        return self.normal(b, heads, tokens, d)

    def outliers(self, x, heads):
        """x [..., heads, tokens, dim] with four channels of each head six times as large."""
        at = torch.rand((heads, 1, self.case["dim"]), generator=self.g, device="cuda").topk(4, dim=2).indices
        return x.mul_(torch.ones((heads, 1, self.case["dim"]), device="cuda", dtype=x.dtype).scatter_(2, at, 6.0))


def _pool(case, m, st, held):
    """Pages in no order and what the sequences hold in them, 8-bit pages as codes and scales."""
    b, h, d, p = case["batch"], case["kv_heads"], case["dim"], case["page"]
    each = (held + p - 1) // p
    total = int(each.sum()) + 3
    order = torch.randperm(total, generator=m.g, device="cuda").to(torch.int32)
    table = torch.full((b, int(case["hi"] + p - 1) // p), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(table.shape[1]) < each[:, None]
    table[used.cuda()] = order[: int(each.sum())]
    st["table"] = table
    st["k_pages"], st["v_pages"] = m.outliers(m.normal(total, h, p, d), h), m.normal(total, h, p, d)
    if case["store"] == "e4m3":
        for x in "kv":
            pages = st[x + "_pages"]
            st[x + "_scale"] = s = _power(pages.abs().amax((2, 3)).float())
            st[x + "_pages"] = (pages.float() / s[:, :, None, None]).to(_E4M3)
            del pages


def prepare(case, seed):
    m = _Maker(case, seed)
    b, h, g, d, n = case["batch"], case["kv_heads"], case["group"], case["dim"], case["hi"]
    held, new = _lengths(case)
    st = {"case": case, "len": held.to("cuda", torch.int32), "new": new.to("cuda", torch.int32)}
    if case["op"] != "cross":
        _pool(case, m, st, held)
    if case["op"] == "append":
        st["k"], st["v"] = m.outliers(m.rows(h, case["new_hi"]), h), m.rows(h, case["new_hi"])
        st["freq"] = _frequencies(case).cuda()
        first = (held - new) // case["page"]  # the pages that the new rows go to, as the program that gave them out knows them
        st["seq"] = torch.repeat_interleave(torch.arange(b), (held - 1) // case["page"] - first + 1).cuda()
        st["at"] = torch.cat([torch.arange(int(a), int(z) + 1) for a, z in zip(first, (held - 1) // case["page"])]).cuda()
    elif case["op"] == "read":
        st["first"] = (st["len"] * case["skip"] // 1000).to(torch.int32)
        st["k_out"], st["v_out"] = (torch.zeros((b, h, n, d), device="cuda", dtype=_DT[case["dtype"]]) for _ in "kv")
    else:
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, h * g + 1, device="cuda") / (h * g)) if case["slopes"] else None
    if case["op"] == "attend":
        st["q"], st["out"] = m.normal(b, h * g, d), torch.zeros((b, h * g, d), device="cuda")
        st["first"] = (st["len"].long() * case["docs"] // 1000).to(torch.int32) if case["docs"] else None
    elif case["op"] == "cross":
        st["q"], st["k"], st["v"] = m.rows(h * g, case["new_hi"]), m.outliers(m.rows(h, n), h), m.rows(h, n)
        st["out"] = torch.zeros((b, h * g, case["new_hi"], d), device="cuda", dtype=st["q"].dtype)
        st["q_pos"] = (st["len"] - st["new"]) if case["causal"] else None
    if own:
        from paper_2412_16187_b200 import HashEvictCache, PagedCache, Rotary, ScoreMod

        if case["op"] == "cross":
            st["cache"] = c = HashEvictCache(b, h, g, d, 32, torch.full((b,), 16), torch.zeros((d, 32)), dtype=_DT[case["dtype"]])
            st["workspace"] = c.cross_workspace(case["new_hi"], n)
        else:
            st["cache"] = c = PagedCache(b, h, g, d, st["table"], st["k_pages"].shape[0], case["page"], dtype=_DT[case["dtype"]], eight_bit=case["store"] == "e4m3",
                                         length=st["len"])
            for x in ("k_pages", "v_pages", "k_scale", "v_scale"):
                if x in st:
                    getattr(c, x).copy_(st[x])
        if case["op"] == "append":
            st["rotary"] = Rotary(d, base=500000.0, interleaved=case["rot"] == "inter") if case["rot"] != "none" else None
        elif case["op"] != "read":
            st["mod"] = ScoreMod(softcap=case["cap"], window=case["window"], slopes=st["slopes"])
        if case["op"] == "attend":
            st["workspace"] = c.workspace()
    return st


# -------------------------------------------------------------------------------------------------------------------- run
def run(st):
    op = st["case"]["op"]
    if own:
        c = st["cache"]
        if op == "append":
            c.append(st["k"], st["v"], st["new"], rotary=st["rotary"])
            return (c.k_pages, c.v_pages) + ((c.k_scale, c.v_scale) if st["case"]["store"] == "e4m3" else ())
        if op == "attend":
            return c.attend(st["q"], st["mod"], first_pos=st["first"], out=st["out"], workspace=st["workspace"])
        if op == "read":
            return c.read(st["case"]["hi"], first=st["first"], k_out=st["k_out"], v_out=st["v_out"])
        return c.attend_cross(st["q"], st["k"], st["v"], st["new"], st["len"], q_pos=st["q_pos"], mod=st["mod"], out=st["out"], workspace=st["workspace"])
    return {"append": _run_append, "attend": _run_attend, "read": _run_read, "cross": _run_cross}[op](st)


def _power(top):
    """The least power of two s >= 2^-100 with top <= 448 s; 2^-100 where there is nothing."""
    part, e = torch.frexp(top)  # top = part 2^e, part in [1/2, 1); 448 = 0.875 2^9
    return torch.ldexp(torch.ones_like(top), torch.where(top > 0, torch.where(part > 0.875, e - 8, e - 9).clamp(min=-100), -100))


def _rotated(st, x, pos):
    """Rows x [..., dim] by the positions pos (one axis fewer), in the dtype of x. Angles in 64 bits, the rotation in 32."""
    if st["case"]["rot"] == "none":
        return x
    angle = pos[..., None] * st["freq"]
    cos, sin, y = angle.cos().float(), angle.sin().float(), x.float()
    if st["case"]["rot"] == "inter":
        a, c = y[..., 0::2], y[..., 1::2]
        return torch.stack((a * cos - c * sin, c * cos + a * sin), dim=-1).flatten(-2).to(x.dtype)
    a, c = y.chunk(2, dim=-1)
    return torch.cat((a * cos - c * sin, c * cos + a * sin), dim=-1).to(x.dtype)


def _run_append(st):
    case, p = st["case"], st["case"]["page"]
    pos = st["at"][:, None] * p + torch.arange(p, device="cuda")
    first = (st["len"] - st["new"]).long()[st["seq"], None]
    row = pos - first
    fresh = ((row >= 0) & (pos < st["len"][st["seq"], None]))[:, None, :, None]
    row = row.clamp(0, case["new_hi"] - 1)
    page = st["table"][st["seq"], st["at"]].long()
    found = []
    for x in "kv":
        rows = st[x].transpose(1, 2)[st["seq"][:, None], row]  # [touched pages, tokens, heads, dim]
        rows = (_rotated(st, rows, pos[:, :, None]) if x == "k" else rows).transpose(1, 2)
        pages = st[x + "_pages"]
        if case["store"] == "same":
            pages[page] = torch.where(fresh, rows, pages[page])
        else:
            scale, rows, old = st[x + "_scale"], rows.float(), pages.view(torch.uint8)[page].view(_E4M3).float()
            need = _power(torch.where(fresh, rows.abs(), 0.0).amax((2, 3)))
            s = torch.where(pos[:, :1] < first, torch.maximum(need, scale[page]), need)
            code = torch.where(fresh, rows / s[:, :, None, None], old * (scale[page] / s)[:, :, None, None]).to(_E4M3)
            keep = pos[:, None, :, None] < st["len"][st["seq"], None, None, None]  # rows behind the end stay as they are
            pages.view(torch.uint8)[page] = torch.where(keep, code.view(torch.uint8), pages.view(torch.uint8)[page])
            scale[page] = s
        found.append(pages)
    return tuple(found) + ((st["k_scale"], st["v_scale"]) if case["store"] == "e4m3" else ())


def _rows_of(st, x):
    """What the pages hold, [batch, heads, tokens, dim] in 32 bits (anything behind a sequence's end)."""
    case, table = st["case"], st["table"].clamp(min=0).long()
    b, n = table.shape
    pages = st[x + "_pages"]
    rows = pages[table] if case["store"] == "same" else pages.view(torch.uint8)[table].view(_E4M3)
    rows = rows.float()
    if case["store"] == "e4m3":
        rows = rows * st[x + "_scale"][table][..., None, None]
    return rows.transpose(1, 2).reshape(b, case["kv_heads"], n * case["page"], case["dim"])


def _run_read(st):
    n, found = st["case"]["hi"], []
    at = st["first"].long()[:, None] + torch.arange(n, device="cuda")
    inside = (at < st["len"][:, None])[:, None, :, None]
    for x in "kv":
        rows = _rows_of(st, x)
        rows = rows.gather(2, at.clamp(max=rows.shape[2] - 1)[:, None, :, None].expand(-1, rows.shape[1], -1, rows.shape[3]))
        found.append(torch.where(inside, rows.to(st[x + "_out"].dtype), st[x + "_out"]))
    return tuple(found)


def _weighted(s, seen, v):
    """softmax(s) v over the keys that `seen` leaves to a row; zeros where it leaves none. s is used up."""
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(dim=-1, keepdim=True)
    b, hq, rows, n = s.shape
    o = (s.reshape(b, v.shape[1], -1, n) @ v.float()).reshape(b, hq, rows, -1)
    return torch.where(total > 0, o / total, 0.0)


def _scores(st, q, k):
    """[batch, query heads, rows, keys] of q [batch, query heads, rows, dim] and k [batch, KV heads, keys, dim], capped."""
    b, hq, rows, d = q.shape
    s = q.float().reshape(b, k.shape[1], -1, d) @ k.float().transpose(2, 3)
    s = s.reshape(b, hq, rows, -1).mul_(d ** -0.5)
    cap = st["case"]["cap"]
    return s.div_(cap).tanh_().mul_(cap) if cap else s


def _run_attend(st):
    case, k = st["case"], _rows_of(st, "k")
    s = _scores(st, st["q"][:, :, None], k)
    j, now = torch.arange(k.shape[2], device="cuda"), st["len"].long()[:, None] - 1
    if case["slopes"]:
        s.sub_((st["slopes"][:, None] * (now - j)[:, None])[:, :, None])
    seen = j <= now
    if case["window"]:
        seen = seen & (j > now - case["window"])
    if case["docs"]:
        seen = seen & (j >= st["first"][:, None])
    v = torch.where((j <= now)[:, None, :, None], _rows_of(st, "v"), 0.0)
    return _weighted(s, seen[:, None, None], v)[:, :, 0]


def _run_cross(st):
    case, n = st["case"], st["k"].shape[2]
    s = _scores(st, st["q"], st["k"])
    i, j = torch.arange(st["q"].shape[2], device="cuda"), torch.arange(n, device="cuda")
    seen = (j < st["len"][:, None])[:, None]
    if case["causal"]:
        away = (st["q_pos"][:, None] + i)[:, :, None] - j  # [batch, rows, keys]
        seen = seen & (away >= 0)
        if case["window"]:
            seen = seen & (away < case["window"])
        if case["slopes"]:
            s.sub_(st["slopes"][:, None, None] * away.abs()[:, None])
    o = _weighted(s, seen[:, None], st["v"])
    return torch.where((i < st["new"][:, None])[:, None, :, None], o.to(st["q"].dtype), st["out"])


# ------------------------------------------------------------------------------------------------------------------- work
def work(case):
    e, d, g, h, b = 4 if case["dtype"] == "f32" else 2, case["dim"], case["group"], case["kv_heads"], case["batch"]
    held, new = _lengths(case)
    stored = 1 if case.get("store") == "e4m3" else e
    if case["op"] == "append":  # every row in and out; the rotation's products and sums
        rows = int(new.sum()) * h
        return {"bytes": 2 * rows * d * (e + stored), "flops": rows * d * (0 if case["rot"] == "none" else 3)}
    if case["op"] == "read":
        rows = int((held - held * case["skip"] // 1000).sum()) * h
        return {"bytes": 2 * rows * d * (e + stored), "flops": 0}
    if case["op"] == "attend":  # the rows that the token sees, the queries in, the outputs out in 32 bits
        low = held * case["docs"] // 1000
        if case["window"]:
            low = torch.maximum(low, held - case["window"])
        seen = int((held - low).sum()) * h
        return {"bytes": seen * 2 * d * stored + b * h * g * d * (e + 4), "flops": seen * g * 4 * d}
    pairs, keys = 0, 0
    for n, r in zip(held.tolist(), new.tolist()):
        t = torch.arange(n - r, n) if case["causal"] else torch.full((r,), n - 1)
        low = (t - case["window"] + 1).clamp(min=0) if case["window"] else torch.zeros_like(t)
        pairs += int((t + 1 - low).sum())
        keys += n - int(low.min())
    return {"bytes": (2 * int(new.sum()) * g + 2 * keys) * h * d * e, "flops": pairs * h * g * 4 * d}


# ------------------------------------------------------------------------------------------------------------------ exact
def _turned(case, x, pos):
    """Rows x [heads, tokens, dim] by their positions in 64 bits: the pairs as complex numbers."""
    y = x.double()
    if case["rot"] == "none":
        return y
    turn = torch.polar(torch.ones_like(pos, dtype=torch.float64)[:, None], pos.double()[:, None] * _frequencies(case).cuda())
    two = (y.unflatten(-1, (-1, 2)) if case["rot"] == "inter" else y.unflatten(-1, (2, -1)).transpose(-1, -2)).contiguous()
    two = torch.view_as_real(torch.view_as_complex(two) * turn)
    return (two if case["rot"] == "inter" else two.transpose(-1, -2)).flatten(-2)


def _exact_append(case, st, held, new):
    """Pages before the last rounding to 8 bits (codes as real numbers); the scales follow from rows rounded to the dtype and are given as they are."""
    p, found = case["page"], {}
    for x in "kv":
        found[x] = st[x + "_pages"].double()
        found[x + "s"] = st[x + "_scale"].double() if case["store"] == "e4m3" else None
    for s in range(case["batch"]):
        n, first = int(held[s]), int(held[s] - new[s])
        rows = {"k": _turned(case, st["k"][s, :, : n - first], torch.arange(first, n, device="cuda")), "v": st["v"][s, :, : n - first].double()}
        for at in range(first // p, (n - 1) // p + 1):
            page, lo, hi = int(st["table"][s, at]), max(at * p, first), min(at * p + p, n)
            for x in "kv":
                y = rows[x][:, lo - first: hi - first]
                if case["store"] == "e4m3":
                    top = y.to(_DT[case["dtype"]]).abs().amax((1, 2)).double()
                    scale = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(min=-100))
                    if lo > at * p:
                        scale = torch.maximum(scale, found[x + "s"][page])
                        found[x][page, :, : lo - at * p] *= (found[x + "s"][page] / scale)[:, None, None]
                    found[x + "s"][page] = scale
                    y = y / scale[:, None, None]
                found[x][page, :, lo - at * p: hi - at * p] = y
    return (found["k"], found["v"]) + ((found["ks"], found["vs"]) if case["store"] == "e4m3" else ())


def _exact_rows(case, st, x, s, n):
    """The first n rows of sequence s, [heads, n, dim]."""
    ids = st["table"][s, : (n + case["page"] - 1) // case["page"]].long()
    if case["store"] == "e4m3":
        y = st[x + "_pages"].view(torch.uint8)[ids].view(_E4M3).double() * st[x + "_scale"][ids].double()[:, :, None, None]
    else:
        y = st[x + "_pages"][ids].double()
    return y.transpose(0, 1).flatten(1, 2)[:, :n]


def exact(case, seed):
    st = prepare(case, seed)
    held, new = _lengths(case)
    h, g, d = case["kv_heads"], case["group"], case["dim"]
    if case["op"] == "append":
        return _exact_append(case, st, held, new) if int(new.sum()) <= 4000 * case["page"] else None  # (page by page)
    if case["op"] == "read":
        found = tuple(st[x + "_out"].double() for x in "kv")
        for s in range(case["batch"]):
            n, first = int(held[s]), int(st["first"][s])
            for x, o in zip("kv", found):
                o[s, :, : n - first] = _exact_rows(case, st, x, s, n)[:, first:]
        return found
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    for s in range(case["batch"]):
        n, r = int(held[s]), int(new[s])
        if case["op"] == "attend":
            k, v, r = _exact_rows(case, st, "k", s, n), _exact_rows(case, st, "v", s, n), 1
        else:
            k, v = st["k"][s, :, :n].double(), st["v"][s, :, :n].double()
        t = torch.arange(n - r, n, device="cuda")[:, None]
        p = torch.arange(n, device="cuda")[None]
        for w in range(h * g):
            rows = st["q"][s, w][None].double() if case["op"] == "attend" else st["q"][s, w, :r].double()
            x = rows @ k[w // g].T / math.sqrt(d)
            if case["cap"]:
                x = torch.tanh(x / case["cap"]) * case["cap"]
            if case["slopes"]:
                x = x - st["slopes"][w].double() * (t - p).abs()
            hide = p > t if case.get("causal", True) else torch.zeros_like(x, dtype=torch.bool)
            if case["window"]:
                hide = hide | (t - p >= case["window"])
            if case.get("docs"):
                hide = hide | (p < st["first"][s])
            x = torch.where(hide, -math.inf, x)
            y = torch.nan_to_num(torch.exp(x - torch.logsumexp(x, 1, keepdim=True)), nan=0.0) @ v[w // g]
            if case["op"] == "attend":
                out[s, w] = y[0]
            else:
                out[s, w, :r] = y
    return out
