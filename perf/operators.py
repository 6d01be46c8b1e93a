"""What is measured of the operators around the compressed cache: rotary positions for the rows that enter it, and attention
whose scores are capped, biased by distance and masked, over a prompt and, token by token, over the cache.

A case is a flat dict:
  op        "rotate_prompt": q and k rows of a batch of prompts, rotated by their positions
            "rotate_step": q and k of one new token per sequence, rotated by the position that the cache holds for it
            "attend_prompt": attention of prompts over themselves
            "attend_scored": attention of one new token per sequence over its compressed cache
  batch, kv_heads, group, dim, dtype      shape of a layer; all the calls take bf16 or f32
  lo, hi    prompt lengths (cache budgets for the single-token calls), uniform in that range, a sequence each
  layout    "heads": [batch, heads, tokens, dim] in memory, "tokens": [batch, tokens, heads, dim], as a projection leaves them
rotary: rot (rotated channels of a row), pairs ("half" or "inter"), base, scaling ("none", "linear", "ntk", "yarn", "bands"),
  factor, offset (position of the first token)
attention: cap (tanh cap of the scores, 0: none), slopes (distance bias), window (0: none), docs (mean length of the documents
  packed into a prompt, 0: one; for the single-token call the share, in thousandths, of the positions that belong to earlier
  documents), prefix (thousandths of a prompt that all its tokens see)
"""
import math

import torch

own = False
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------------ cases
def _shape(name, op, batch, kv_heads, group, dim, dtype, lo, hi, layout="heads"):
    return {"name": name, "op": op, "batch": batch, "kv_heads": kv_heads, "group": group, "dim": dim, "dtype": dtype, "lo": lo, "hi": hi,
            "layout": layout}


def _rotary(name, op, *shape, rot, pairs="half", base=10000.0, scaling="none", factor=1.0, offset=0, layout="heads"):
    return {**_shape(name, op, *shape, layout=layout), "rot": rot, "pairs": pairs, "base": base, "scaling": scaling, "factor": factor, "offset": offset}


def _attend(name, op, *shape, cap=0.0, slopes=False, window=0, docs=0, prefix=0, layout="heads"):
    return {**_shape(name, op, *shape, layout=layout), "cap": cap, "slopes": slopes, "window": window, "docs": docs, "prefix": prefix}


def listed():
    return [
        # --- rotary positions
        # one token of the tiny configuration: nothing but the latency of a call
        _rotary("rotate step tiny fp32", "rotate_step", 1, 4, 1, 64, "f32", 64, 64, rot=64),
        # one token of each of 256 sequences far into their texts, a long-context layer's frequencies
        _rotary("rotate step x256, far", "rotate_step", 256, 8, 4, 128, "bf16", 512, 4096, rot=128, base=500000.0, scaling="bands", factor=8.0,
                offset=100000),
        # ragged prompts of the throughput batch straight from the projection, a quarter of each head rotated in neighbouring pairs
        _rotary("rotate ragged x16, part", "rotate_prompt", 16, 8, 4, 128, "bf16", 1024, 8192, rot=32, pairs="inter", layout="tokens"),
        # one layer of a long-context prompt, frequencies stretched by parts
        _rotary("rotate long layer", "rotate_prompt", 1, 8, 4, 128, "bf16", 32768, 32768, rot=128, scaling="yarn", factor=8.0),
        # --- attention of a prompt over itself
        # the tiny configuration in fp32, capped scores
        _attend("prompt tiny fp32, cap", "attend_prompt", 1, 4, 1, 64, "f32", 128, 128, cap=30.0),
        # a multi-head layer of a 4096-token prompt, capped scores
        _attend("prompt mha layer, cap", "attend_prompt", 1, 32, 1, 128, "bf16", 4096, 4096, cap=30.0),
        # ragged prompts packed from documents, bias by distance, rows as the projection leaves them
        _attend("prompt gqa x4, docs + bias", "attend_prompt", 4, 8, 4, 128, "bf16", 1024, 4096, slopes=True, docs=700, layout="tokens"),
        # a prefix that all tokens see, heads of 64, odd lengths
        _attend("prompt x8 d64, prefix", "attend_prompt", 8, 8, 2, 64, "bf16", 501, 2777, prefix=300),
        # one KV head's share of a long-context prompt
        _attend("prompt long", "attend_prompt", 1, 1, 4, 128, "bf16", 32768, 32768),
        # --- attention of a new token over the compressed cache
        _attend("cache tiny fp32, bias", "attend_scored", 1, 4, 1, 64, "f32", 64, 64, slopes=True),
        # long context at batch 1: 9830 slots per head, bias by distance within a window
        _attend("cache long, bias + window", "attend_scored", 1, 8, 4, 128, "bf16", 9830, 9830, slopes=True, window=12000),
        # the throughput batch: 64 sequences with ragged budgets, capped scores, the earlier documents hidden
        _attend("cache ragged x64, cap + doc", "attend_scored", 64, 8, 4, 128, "bf16", 512, 4096, cap=30.0, docs=250),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Shapes of a transformer layer (1 to 32 KV heads, groups of 1 to 8, heads of 64 to 128), prompts of one token to 32768,
    budgets to 9830, and every combination of the options that a call takes."""
    while True:
        op = rng.choice(("rotate_step", "rotate_prompt", "attend_prompt", "attend_prompt", "attend_scored"))
        dtype = "f32" if rng.random() < 0.15 else "bf16"
        dim = rng.choice((64, 80, 96, 128, 128, 128))
        heads, group = rng.choice((1, 2, 4, 8, 8, 32)), rng.choice((1, 2, 4, 4, 4, 7, 8))
        layout = rng.choice(("heads", "tokens"))
        if op.startswith("rotate"):
            batch, hi = _log(rng, 1, 256), _log(rng, 1, 32768) if op == "rotate_prompt" else 64
            lo = rng.randint(max(1, hi // 8), hi)
            rot = rng.choice((dim, dim, dim // 2, dim // 4))
            scaling = rng.choice(("none", "linear", "ntk", "yarn", "bands"))
            c = _rotary("", op, batch, heads, group, dim, dtype, lo, hi, rot=rot, pairs=rng.choice(("half", "inter")),
                        base=rng.choice((10000.0, 500000.0)), scaling=scaling, factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)),
                        offset=rng.choice((0, 0, _log(rng, 1, 1000000))), layout=layout)
            if batch * hi * heads * (group + 1) * dim > 16 * 8192 * 8 * 5 * 128:
                continue
        elif op == "attend_prompt":
            batch, hi = _log(rng, 1, 32), _log(rng, 1, 32768)
            lo = rng.randint(max(1, hi // 8), hi)
            c = _attend("", op, batch, heads, group, dim, dtype, lo, hi, cap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.4,
                        window=rng.choice((0, 0, _log(rng, 16, 8192))), docs=rng.choice((0, 0, _log(rng, 32, 4096))),
                        prefix=rng.choice((0, 0, rng.randint(1, 1000))), layout=layout)
            if batch * heads * group * hi * hi > 4 * 32768 * 32768 // (1 if dtype == "bf16" else 16):
                continue
        else:
            batch, hi = _log(rng, 1, 64), _log(rng, 16, 9830)
            lo = rng.randint(max(8, hi // 8), hi)
            c = _attend("", op, batch, heads, group, dim, dtype, lo, hi, cap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.4,
                        window=rng.choice((0, 0, _log(rng, 16, 8192))), docs=rng.choice((0, 0, rng.randint(1, 900))))
            if batch * heads * hi * dim * (2 if dtype == "f32" else 1) > 64 * 8 * 2304 * 128 or batch * heads * group * hi > 64 * 8 * 4 * 4096:
                continue
        del c["name"]
        return c


def _lengths(case):
    """Prompt lengths or budgets of the sequences. Part of the case: two seeds of it differ in values only."""
    g = torch.Generator().manual_seed(case["lo"] * 1_000_003 + case["hi"])
    return torch.randint(case["lo"], case["hi"] + 1, (case["batch"],), generator=g)


def _doc_starts(case):
    """First position of the document that each token of a prompt belongs to, [batch, tokens]; part of the case too."""
    g = torch.Generator().manual_seed(case["docs"] * 7 + case["hi"])
    cut = torch.rand((case["batch"], case["hi"]), generator=g) < 1.0 / case["docs"]
    at = torch.arange(case["hi"]).expand(case["batch"], -1)
    return torch.where(cut, at, 0).cummax(1).values.to(torch.int32)


def _frequencies(case):
    """Radians per position of each pair and the factor on both components, in 64 bits."""
    r, base, f = case["rot"], case["base"], case["factor"]
    i = torch.arange(r // 2, dtype=torch.float64)
    if case["scaling"] == "ntk":
        base = base * f ** (r / (r - 2))
    freq = base ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return freq / f, 1.0
    if case["scaling"] == "yarn":  # pairs that turn fewer than once in 8192 positions are stretched, those of over 32 turns are not
        low, high = (r * math.log(8192 / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (32.0, 1.0))
        low, high = max(math.floor(low), 0), min(math.ceil(high), r - 1)
        ramp = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
        return freq / f * ramp + freq * (1 - ramp), 0.1 * math.log(f) + 1.0
    if case["scaling"] == "bands":
        turns = 8192 * freq / (2 * math.pi)
        smooth = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return (1 - smooth) * freq / f + smooth * freq, 1.0
    return freq, 1.0


def _scaling(case):
    k = {"none": None, "linear": {}, "ntk": {}, "yarn": {"length": 8192}, "bands": {"length": 8192, "low": 1.0, "high": 4.0}}[case["scaling"]]
    return None if k is None else {"kind": case["scaling"], "factor": case["factor"], **k}


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
        if self.case["layout"] == "tokens":
            return self.normal(b, tokens, heads, d).transpose(1, 2)
        return self.normal(b, heads, tokens, d)

    def keys(self, heads, tokens):
        x = self.rows(heads, tokens)
        at = torch.rand((self.case["batch"], heads, 1, self.case["dim"]), generator=self.g, device="cuda").topk(4, dim=3).indices
        return x.mul_(torch.ones_like(x[:, :, :1]).scatter_(3, at, 6.0))


def prepare(case, seed):
    m = _Maker(case, seed)
    b, h, g, d = case["batch"], case["kv_heads"], case["group"], case["dim"]
    lens, n = _lengths(case), case["hi"]
    st = {"case": case, "len": lens.to("cuda", torch.int32)}
    if case["op"].startswith("rotate"):
        st["freq"], st["amp"] = _frequencies(case)
        st["freq"] = st["freq"].cuda()
        tokens = n if case["op"] == "rotate_prompt" else 1
        st["q"], st["k"] = m.rows(h * g, tokens), m.keys(h, tokens)
        st["q_out"], st["k_out"] = torch.zeros((b, h * g, tokens, d), device="cuda", dtype=st["q"].dtype), torch.zeros((b, h, tokens, d), device="cuda", dtype=st["q"].dtype)
        if tokens == 1 and case["op"] == "rotate_step":
            st.update({x: st[x][:, :, 0].contiguous() for x in ("q", "k")}, **{x: st[x][:, :, 0] for x in ("q_out", "k_out")})
            st["next_pos"] = (case["offset"] + 2 * st["len"])[:, None].expand(b, h).contiguous()
        else:
            st["pos"] = (case["offset"] + torch.arange(n, device="cuda", dtype=torch.int32)).expand(b, n).contiguous() if case["offset"] else None
    else:
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, h * g + 1, device="cuda") / (h * g)) if case["slopes"] else None
        if case["op"] == "attend_prompt":
            st["q"], st["k"], st["v"] = m.rows(h * g, n), m.keys(h, n), m.rows(h, n)
            st["out"] = torch.zeros((b, h * g, n, d), device="cuda", dtype=st["q"].dtype)
            st["doc"] = _doc_starts(case).cuda() if case["docs"] else None
            st["prefix"] = (st["len"] * case["prefix"] // 1000) if case["prefix"] else None
        else:
            # a cache as the eviction leaves it: each sequence has seen twice its budget, the newest token and a random choice of
            # the others are resident, in no order
            seen, slots = 2 * n, (n + 3) // 4 * 4
            st["q"], st["out"] = m.normal(b, h * g, d), torch.zeros((b, h * g, d), device="cuda")
            st["k"], st["v"] = m.keys(h, slots).contiguous(), m.normal(b, h, slots, d)
            order = torch.rand((b, h, seen), generator=m.g, device="cuda")
            at = torch.arange(seen, device="cuda")
            last = (2 * st["len"].long() - 1)[:, None, None]
            order = torch.where(at > last, 2.0, torch.where(at == last, -1.0, order))
            order = order.argsort(dim=2)[:, :, :slots]
            where = torch.rand((b, h, slots), generator=m.g, device="cuda")
            where = torch.where(torch.arange(slots, device="cuda") < st["len"][:, None, None], where, 2.0).argsort(dim=2)  # shuffles the valid ones
            pos = order.gather(2, where).to(torch.int32)
            st["slot_pos"] = torch.where(torch.arange(slots, device="cuda") < st["len"][:, None, None], pos, -1)
            st["fill"] = st["len"][:, None].expand(b, h).contiguous()
            st["next_pos"] = 2 * st["fill"]
            st["first"] = (2 * st["len"].long() * case["docs"] // 1000).to(torch.int32) if case["docs"] else None
    if own:
        from paper_2412_16187_b200 import HashEvictCache, Rotary, ScoreMod

        budgets = lens if case["op"] == "attend_scored" else torch.full((b,), 16)
        st["cache"] = c = HashEvictCache(b, h, g, d, 32, budgets, torch.zeros((d, 32)), dtype=_DT[case["dtype"]], max_budget=int(n) if case["op"] == "attend_scored" else None)
        if "next_pos" in st:
            c.next_pos.copy_(st["next_pos"])
        if case["op"].startswith("rotate"):
            st["rotary"] = Rotary(d, case["rot"], base=case["base"], interleaved=case["pairs"] == "inter", scaling=_scaling(case))
        else:
            st["mod"] = ScoreMod(softcap=case["cap"], window=case["window"], slopes=st["slopes"])
        if case["op"] == "attend_scored":
            for mine, theirs in (("k_cache", "k"), ("v_cache", "v"), ("pos", "slot_pos"), ("fill", "fill")):
                getattr(c, mine).copy_(st[theirs])
    return st


# -------------------------------------------------------------------------------------------------------------------- run
def run(st):
    op = st["case"]["op"]
    if own:
        c = st["cache"]
        if op == "rotate_prompt":
            return c.rotate_prompt(st["rotary"], st["q"], st["k"], st["len"], positions=st["pos"], q_out=st["q_out"], k_out=st["k_out"])
        if op == "rotate_step":
            return c.rotate_step(st["rotary"], st["q"], st["k"], q_out=st["q_out"], k_out=st["k_out"])
        if op == "attend_prompt":
            return c.attend_prompt(st["q"], st["k"], st["v"], st["len"], mod=st["mod"], doc_start=st["doc"], prefix_len=st["prefix"], out=st["out"])
        return c.attend_scored(st["q"], st["mod"], first_pos=st["first"], out=st["out"])
    if op == "rotate_prompt":
        at = torch.arange(st["q"].shape[2], device="cuda")
        past = (at >= st["len"][:, None])[:, None, :, None]  # rows behind a prompt's end are left as they were
        pos = st["pos"] if st["pos"] is not None else at.expand(st["len"].shape[0], -1)
        return tuple(torch.where(past, st[x + "_out"], _rotated(st, st[x], pos[:, None])) for x in "qk")
    if op == "rotate_step":
        g = st["case"]["group"]
        return _rotated(st, st["q"], st["next_pos"].repeat_interleave(g, dim=1)), _rotated(st, st["k"], st["next_pos"])
    return _attend_prompt(st) if op == "attend_prompt" else _attend_scored(st)


def _rotated(st, x, pos):
    """Rows x by the positions pos (one axis fewer). Angles in 64 bits, the rotation in 32."""
    r, angle = st["case"]["rot"], pos[..., None] * st["freq"]
    cos, sin = (angle.cos() * st["amp"]).float(), (angle.sin() * st["amp"]).float()
    y, rest = x[..., :r].float(), x[..., r:]
    if st["case"]["pairs"] == "inter":
        a, c = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * cos - c * sin, c * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, c = y[..., : r // 2], y[..., r // 2:]
        y = torch.cat((a * cos - c * sin, c * cos + a * sin), dim=-1)
    return torch.cat((y.to(x.dtype), rest), dim=-1)


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


def _attend_prompt(st):
    case, n = st["case"], st["q"].shape[2]
    s = _scores(st, st["q"], st["k"])
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")
    if case["slopes"]:
        s.sub_(st["slopes"][:, None, None] * (i - j).abs())
    low, high = torch.zeros_like(i)[None], (i + 1)[None]
    if case["docs"]:
        low = st["doc"][:, :, None]
    if case["window"]:
        low = torch.maximum(low, i - case["window"] + 1)
    if case["prefix"]:
        high = torch.maximum(high, st["prefix"][:, None, None])
    seen = (j >= low) & (j < torch.minimum(high, st["len"][:, None, None]))
    o = _weighted(s, seen[:, None], st["v"])
    return torch.where((i < st["len"][:, None, None])[:, None], o.to(st["q"].dtype), st["out"])


def _attend_scored(st):
    case, pos = st["case"], st["slot_pos"]
    b, h, slots = pos.shape
    s = _scores(st, st["q"][:, :, None], st["k"])
    now = st["next_pos"][:, :, None] - 1
    if case["slopes"]:
        s.sub_((st["slopes"].view(h, -1, 1) * (now - pos)[:, :, None]).view(b, -1, 1, slots))
    seen = torch.arange(slots, device="cuda") < st["fill"][:, :, None]
    if case["window"]:
        seen = seen & (pos > now - case["window"])
    if case["docs"]:
        seen = seen & (pos >= st["first"][:, None, None])
    return _weighted(s, seen.repeat_interleave(case["group"], dim=1)[:, :, None], st["v"])[:, :, 0]


# ------------------------------------------------------------------------------------------------------------------- work
def _span(case):
    """How many keys each token of each prompt sees, summed over the batch."""
    lens, n = _lengths(case), case["hi"]
    i = torch.arange(n)
    low = _doc_starts(case).long() if case["docs"] else torch.zeros((case["batch"], n), dtype=torch.int64)
    if case["window"]:
        low = torch.maximum(low, i - case["window"] + 1)
    high = (i + 1).expand(case["batch"], n)
    if case["prefix"]:
        high = torch.maximum(high, (lens * case["prefix"] // 1000)[:, None])
    high = torch.minimum(high, lens[:, None])
    return int(((high - low).clamp(min=0) * (i < lens[:, None])).sum())


def work(case):
    e, d, g, h, b = 4 if case["dtype"] == "f32" else 2, case["dim"], case["group"], case["kv_heads"], case["batch"]
    tokens = int(_lengths(case).sum())
    if case["op"].startswith("rotate"):
        # every row in and out; two products and two sums for each rotated pair's components
        rows = (tokens if case["op"] == "rotate_prompt" else b) * h * (g + 1)
        return {"bytes": 2 * rows * d * e, "flops": rows * case["rot"] * 3}
    if case["op"] == "attend_prompt":
        return {"bytes": tokens * h * (2 * g + 2) * d * e, "flops": _span(case) * h * g * 4 * d}
    # K, V and positions of the budgets in, the queries in, the outputs out in 32 bits
    return {"bytes": tokens * h * (2 * d * e + 4) + b * h * g * d * (e + 4), "flops": tokens * h * g * 4 * d}


# ------------------------------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    st = prepare(case, seed)
    b, h, g, d = case["batch"], case["kv_heads"], case["group"], case["dim"]
    if case["op"].startswith("rotate"):
        if case["op"] == "rotate_prompt":
            pos = (case["offset"] + torch.arange(case["hi"], device="cuda")).expand(b, 1, case["hi"])
            inside = torch.arange(case["hi"], device="cuda") < st["len"][:, None, None]
        else:
            pos, inside = st["next_pos"][:, :1], torch.ones((b, 1), dtype=torch.bool, device="cuda")
        turn = torch.polar(torch.full_like(st["freq"], st["amp"]), st["freq"] * pos.double()[..., None])  # the pairs as complex numbers
        r, found = case["rot"], []
        for x in (st["q"], st["k"]):
            y = x.double()
            two = (y[..., :r].unflatten(-1, (-1, 2)) if case["pairs"] == "inter" else y[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)).contiguous()
            two = torch.view_as_real(torch.view_as_complex(two) * turn)
            y[..., :r] = (two if case["pairs"] == "inter" else two.transpose(-1, -2)).flatten(-2)
            found.append(torch.where(inside[..., None], y, 0.0))
        return tuple(found)
    prompt = case["op"] == "attend_prompt"
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    for s in range(b):
        n = int(st["len"][s])
        for u in range(h):
            k, v = st["k"][s, u, :n].double(), st["v"][s, u, :n].double()
            for w in range(u * g, u * g + g):
                for at in range(0, n if prompt else 1, 4096):
                    if prompt:
                        t = torch.arange(at, min(n, at + 4096), device="cuda")[:, None]
                        p, rows = torch.arange(n, device="cuda")[None], st["q"][s, w, at:at + 4096][:n - at].double()
                        hide = (p > t) if st["prefix"] is None else (p > t) & (p >= st["prefix"][s])
                        first = st["doc"][s, at:at + 4096][:n - at, None] if st["doc"] is not None else None
                    else:
                        t, p = st["next_pos"][s, u] - 1, st["slot_pos"][s, u, :n][None]
                        rows, hide, first = st["q"][s, w][None].double(), torch.zeros_like(p, dtype=torch.bool), st["first"][s] if st["first"] is not None else None
                    x = rows @ k.T / math.sqrt(d)
                    if case["cap"]:
                        x = torch.tanh(x / case["cap"]) * case["cap"]
                    if case["slopes"]:
                        x = x - st["slopes"][w].double() * (t - p).abs()
                    if case["window"]:
                        hide = hide | (t - p >= case["window"])
                    if first is not None:
                        hide = hide | (p < first)
                    x = torch.where(hide, -math.inf, x)
                    y = torch.nan_to_num(torch.exp(x - torch.logsumexp(x, 1, keepdim=True)), nan=0.0) @ v  # a row without keys gives zeros
                    if prompt:
                        out[s, w, at:at + 4096][:n - at] = y
                    else:
                        out[s, w] = y[0]
    return out
