"""Attention of rows over keys of another length against its definition in 64 bits, and prompts that come in chunks."""
import math

import pytest
import torch

from layer_reference import attend, tolerance
from paper_2412_16187_b200 import HashEvictCache, HashEvictError, PagedCache, Rotary, ScoreMod, device_error_count
from test_gpu_layer_ops import BF16, F32, make_cache, rows

pytestmark = pytest.mark.gpu


def seen_by(n, m, q_pos, opt, first, prefix):
    """[rows, keys] that a row sees."""
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(m, device="cuda")[None]
    low = torch.zeros_like(i) if first is None else first[:n, None].long().clamp(min=0)
    if q_pos is None:
        return (j >= low).expand(n, m)
    t = i + q_pos
    if opt.get("window"):
        low = torch.maximum(low, t - opt["window"] + 1)
    return (j >= low) & (j < torch.maximum(t + 1, torch.full_like(t, prefix)))


def case(shape, opt, seed=0):
    b, h, g, d, dtype, q_lens, kv_lens, layout = shape
    gen = torch.Generator(device="cuda").manual_seed(seed + d)
    n, m = max(max(q_lens) + 3, 1), max(max(kv_lens) + 5, 1)
    q, k, v = rows(gen, b, h * g, n, d, dtype, layout), rows(gen, b, h, m, d, dtype, layout) * 2, rows(gen, b, h, m, d, dtype, layout)
    kw = {}
    if opt.get("causal"):
        kw["q_pos"] = torch.tensor([y - x + opt.get("shift", 0) for x, y in zip(q_lens, kv_lens)], dtype=torch.int32, device="cuda")
        if "prefix" in opt:
            kw["prefix_len"] = torch.tensor([y * opt["prefix"] // 1000 for y in kv_lens], dtype=torch.int32, device="cuda")
            kw["prefix_len"][-1] = 2 ** 31 - 1
    if "first" in opt:
        kw["first_key"] = torch.randint(0, max(kv_lens) * opt["first"] // 1000 + 1, (b, n), generator=gen, device="cuda").sort(1).values.to(torch.int32)
        kw["first_key"][:, 2::41] = 2 ** 31 - 1  # rows that see nothing
        kw["first_key"][:, 5::43] = -(2 ** 31)
    slopes = torch.exp2(-torch.arange(1, h * g + 1, device="cuda") * 8.0 / (h * g)) if opt.get("slopes") else None
    mod = ScoreMod(scale=opt.get("scale", 0.0), softcap=opt.get("cap", 0.0), window=opt.get("window", 0), slopes=slopes)
    for s in range(b):  # what lies behind the rows and keys may be anything
        q[s, :, q_lens[s]:], k[s, :, kv_lens[s]:], v[s, :, kv_lens[s]:] = math.nan, math.inf, math.nan
    ql, kl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_lens, kv_lens))
    return q, k, v, ql, kl, mod, kw, slopes


def check(out, q, k, v, q_lens, kv_lens, opt, kw, slopes, g, exact_weights):
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        assert bool((out[s, :, n:] == 7.0).all())
        if n == 0:
            continue
        if m == 0:
            assert not out[s, :, :n].any()
            continue
        p = int(kw["q_pos"][s]) if "q_pos" in kw else None
        seen = seen_by(n, m, p, opt, kw["first_key"][s] if "first_key" in kw else None, int(kw["prefix_len"][s]) if "prefix_len" in kw else 0)
        t, at = torch.arange(n, device="cuda") + (p or 0), torch.arange(m, device="cuda")
        for u in range(k.shape[1]):
            sl = slice(u * g, u * g + g)
            ref = attend(q[s, sl, :n], k[s, u, :m], v[s, u, :m], t, at, seen, opt.get("scale", 0.0), opt.get("cap", 0.0), None if slopes is None else slopes[sl])
            got = out[s, sl, :n].double()
            off = (got - ref).abs() - tolerance(ref, v[s, u, :m].double().abs().max(), out.dtype, exact_weights)
            assert bool((off <= 0).all()), (s, u, float(off.max()))
            assert not got[:, ~seen.any(1)].any()


OPTIONS = {
    "all keys": {}, "all keys, cap": {"cap": 20.0}, "all keys, first": {"first": 700, "scale": 0.3}, "causal": {"causal": True}, "causal, cap + bias": {"causal": True, "cap": 5.0, "slopes": True},
    "causal, window": {"causal": True, "window": 37}, "causal, all": {"causal": True, "cap": 30.0, "slopes": True, "first": 500, "prefix": 300, "window": 100},
    "causal, ahead": {"causal": True, "shift": -60, "slopes": True}, "causal, behind": {"causal": True, "shift": 90}, "causal, prefix": {"causal": True, "prefix": 600, "first": 100},
}
# (B, H, G, d, dtype, rows, keys, layout): one row, one key, none of either, more rows than keys, tile edges, few rows over many keys
SHAPES = [
    (1, 2, 2, 64, F32, [40], [200], "heads"), (3, 1, 2, 40, F32, [1, 0, 65], [300, 5, 0], "tokens"), (1, 1, 3, 256, BF16, [20], [700], "heads"), (2, 2, 1, 200, F32, [3, 129], [1100, 63], "heads"),
    (1, 1, 1, 128, BF16, [1], [1], "heads"), (4, 2, 4, 128, BF16, [127, 128, 129, 257], [128, 300, 129, 1], "heads"), (3, 2, 3, 128, BF16, [300, 0, 5], [0, 40, 2000], "tokens"),
    (2, 1, 8, 64, BF16, [1, 1], [3000, 700], "tokens"), (2, 2, 7, 80, BF16, [20, 3], [900, 385], "heads"), (1, 1, 1, 96, BF16, [500], [4000], "tokens"), (2, 2, 2, 8, BF16, [5, 300], [300, 5], "heads"),
    (1, 2, 1, 120, BF16, [256], [1281], "heads"), (8, 4, 1, 64, BF16, [1] * 8, [97 * i for i in range(8)], "heads"), (1, 1, 1, 64, F32, [1], [5000], "heads"),
]
IDS = [f"{'x'.join(map(str, s[:4]))}-{'bf16' if s[4] == BF16 else 'fp32'}-{max(s[5])}-{max(s[6])}" for s in SHAPES]


@pytest.mark.parametrize("opt", list(OPTIONS))
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("path", ["default", "whole", "generic"])
def test_attend_cross(shape, opt, path, monkeypatch):
    b, h, g, d, dtype, q_lens, kv_lens, _ = shape
    tensor_cores = dtype == BF16 and d <= 128
    if path == "generic":
        if not tensor_cores:
            pytest.skip("the default path is already the generic kernel")
        monkeypatch.setenv("HE_DISABLE_ATTEND_MMA", "1")
    o = OPTIONS[opt]
    q, k, v, ql, kl, mod, kw, slopes = case(shape, o)
    cache, out = make_cache(b, h, g, d, dtype), torch.full_like(q, 7.0)
    # "whole": no workspace, a tile walks over all its keys
    ws = torch.empty(0, dtype=torch.uint8, device="cuda") if path == "whole" else torch.full((cache.cross_workspace(q.shape[2], k.shape[2]).numel(),), 255, dtype=torch.uint8, device="cuda")
    assert cache.attend_cross(q, k, v, ql, kl, mod=mod, out=out, workspace=ws, **kw) is out
    check(out, q, k, v, q_lens, kv_lens, o, kw, slopes, g, path == "generic" or not tensor_cores)
    again = torch.full_like(q, 7.0)
    cache.attend_cross(q, k, v, ql, kl, mod=mod, out=again, workspace=ws, **kw)
    assert torch.equal(out, again) and device_error_count() == 0


@pytest.mark.parametrize("opt", ["all keys, cap", "causal, all"])
@pytest.mark.parametrize("shape", [(5, 32, 1, 64, BF16, [130, 300, 0, 1, 260], [5, 300, 40, 0, 300], "heads"), (33, 4, 2, 128, BF16, [40 + 3 * i for i in range(33)], [97 * i % 500 for i in range(33)], "tokens"),
                                   (32, 4, 2, 128, BF16, [136 - 3 * i for i in range(32)], [61 * i % 7 * 80 for i in range(32)], "heads")], ids=["5", "33", "32"])
def test_more_tiles_than_run_at_once(shape, opt):
    """Sequences in the order of their keys (up to 32 of them), equal and empty ones among them."""
    b, h, g, d, dtype, q_lens, kv_lens, _ = shape
    o = OPTIONS[opt]
    q, k, v, ql, kl, mod, kw, slopes = case(shape, o)
    out = make_cache(b, h, g, d, dtype).attend_cross(q, k, v, ql, kl, mod=mod, out=torch.full_like(q, 7.0), workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), **kw)
    check(out, q, k, v, q_lens, kv_lens, o, kw, slopes, g, False)
    assert device_error_count() == 0


@pytest.mark.parametrize("dtype, d", [(BF16, 128), (F32, 64)])
def test_a_prompt_over_itself_is_the_case_of_equal_lengths(dtype, d):
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (rows(gen, 2, x, 400, d, dtype) for x in (8, 2, 2))
    lens = torch.tensor([400, 301], dtype=torch.int32, device="cuda")
    cache, mod = make_cache(2, 2, 4, d, dtype), ScoreMod(softcap=20.0, window=300)
    want, got = torch.zeros_like(q), torch.zeros_like(q)
    cache.attend_prompt(q, k, v, lens, mod=mod, out=want)
    cache.attend_cross(q, k, v, lens, lens, q_pos=torch.zeros_like(lens), mod=mod, out=got, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert torch.equal(got, want)


@pytest.mark.parametrize("shape", [(1, 1, 2, 128, BF16, [30], [1500], "heads"), (1, 2, 1, 64, BF16, [400], [900], "tokens"), (1, 1, 2, 64, F32, [40], [900], "heads")])
@pytest.mark.parametrize("opt", ["all keys, first", "causal", "causal, window", "causal, all"])
@pytest.mark.parametrize("whole", [True, False])
def test_hidden_infinities_and_nans_touch_nobody(shape, opt, whole):
    b, h, g, d, dtype, (n,), (m,), _ = shape
    o = OPTIONS[opt]
    q, k, v, ql, kl, mod, kw, slopes = case(shape, o, seed=5)
    at = [m - n // 2, m // 3]
    clean = v.clone()
    v[0, 0, at[0], 3], v[0, 0, at[0], 5], v[0, 0, at[1], 7] = math.inf, math.nan, -math.inf
    cache = make_cache(b, h, g, d, dtype)
    ws = torch.empty(0, dtype=torch.uint8, device="cuda") if whole else None
    out = cache.attend_cross(q, k, v, ql, kl, mod=mod, workspace=ws, **kw)
    p = int(kw["q_pos"][0]) if "q_pos" in kw else None
    seen = seen_by(n, m, p, o, kw["first_key"][0] if "first_key" in kw else None, int(kw["prefix_len"][0]) if "prefix_len" in kw else 0)
    touched = seen[:, at[0]] | seen[:, at[1]]
    assert bool(torch.isfinite(out[0, :g, :n][:, ~touched]).all())
    t = torch.arange(n, device="cuda") + (p or 0)
    ref = attend(q[0, :g, :n], k[0, 0, :m], clean[0, 0, :m], t, torch.arange(m, device="cuda"), seen, o.get("scale", 0.0), o.get("cap", 0.0), None if slopes is None else slopes[:g])
    tol = tolerance(ref, clean[0, 0, :m].abs().max().double(), dtype, dtype == F32)
    assert bool(((out[0, :g, :n].double() - ref).abs() <= tol)[:, ~touched].all())
    assert not bool(torch.isfinite(out[0, :g, :n][:, seen[:, at[0]]][..., 5]).any())


def test_broadcast_keys_and_streams():
    """Keys of one sequence for all (a stride of zero), another stream, captured and replayed."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    b, h, g, d, n, m = 3, 2, 2, 64, 9, 1300
    q, one_k, one_v = rows(gen, b, h * g, n, d, BF16), rows(gen, 1, h, m, d, BF16), rows(gen, 1, h, m, d, BF16)
    ql, kl = torch.tensor([9, 1, 5], dtype=torch.int32, device="cuda"), torch.tensor([1300, 700, 1], dtype=torch.int32, device="cuda")
    cache = make_cache(b, h, g, d, BF16)
    for k, v in ((one_k.expand(b, -1, -1, -1), one_v.expand(b, -1, -1, -1)), (one_k.repeat(b, 1, 1, 1), one_v.repeat(b, 1, 1, 1))):
        out = torch.full_like(q, 7.0)
        cache.attend_cross(q, k, v, ql, kl, out=out)
        check(out, q, k, v, ql.tolist(), kl.tolist(), {}, {}, None, g, False)
    torch.cuda.synchronize()
    outs, st, graph = [torch.full_like(q, 7.0) for _ in "12"], torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    cache.attend_cross(q, k, v, ql, kl, out=outs[0], stream=st)
    st.synchronize()
    with torch.cuda.graph(graph, stream=st):
        cache.attend_cross(q, k, v, ql, kl, out=outs[1], stream=st)
    graph.replay(), graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], out) and torch.equal(outs[1], out)


def test_the_binding_refuses():
    b, h, g, d = 2, 2, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = make_cache(b, h, g, d, BF16)
    q, k, v = rows(gen, b, h * g, 3, d, BF16), rows(gen, b, h, 7, d, BF16), rows(gen, b, h, 7, d, BF16)
    n = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    for call in (lambda: cache.attend_cross(q, k, v[:, :, :6], n, n), lambda: cache.attend_cross(q, k, v, n.long(), n), lambda: cache.attend_cross(q, k, v, n, n[:1]),
                 lambda: cache.attend_cross(q.float(), k, v, n, n), lambda: cache.attend_cross(q, k, v, n, n, mod=ScoreMod(window=3)), lambda: cache.attend_cross(q, k, v, n, n, prefix_len=n),
                 lambda: cache.attend_cross(q, k, v, n, n, q_pos=n.float()), lambda: cache.attend_cross(q, k, v, n, n, first_key=n), lambda: cache.attend_cross(q, k, v, n, n, out=q),
                 lambda: cache.attend_cross(q, k, k.transpose(1, 2).contiguous().transpose(1, 2), n, n), lambda: cache.attend_cross(q.cpu(), k, v, n, n)):
        with pytest.raises(HashEvictError):
            call()
    big_k = rows(gen, 1, 1, 4000, d, BF16)
    one = make_cache(1, 1, 1, d, BF16)
    with pytest.raises(HashEvictError, match="workspace"):
        one.attend_cross(big_k[:, :, :2], big_k, big_k, n[:1], n[:1], workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert not cache.attend_cross(q, k[:, :, :0], v[:, :, :0], n, n).any()  # no keys at all


@pytest.mark.parametrize("dtype, d, eight", [(BF16, 128, False), (BF16, 64, True), (F32, 64, False)])
def test_a_prompt_in_chunks_then_compressed_then_tokens(dtype, d, eight):
    """A chunk at a time: keys into the pages (rotated on the way), the chunk's rows over all keys so far, read back. Then the whole prompt, from the pages, into the
    compressed cache; then tokens over both caches. In the pages' own dtype everything is what one long prompt gives."""
    b, h, g, n, more, p = 2, 2, 4, 230, 5, 32
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, v = (rows(gen, b, x, n + more, d, dtype) for x in (h * g, h, h))
    w, rot, mod = torch.randn((d, 16), generator=gen, device="cuda"), Rotary(d, d // 2), ScoreMod(softcap=15.0)
    table = torch.randperm(b * 8, generator=gen, device="cuda").to(torch.int32).view(b, 8)
    pages = PagedCache(b, h, g, d, table, b * 8, p, dtype=dtype, eight_bit=eight)
    cache = HashEvictCache(b, h, g, d, 16, [n + more] * b, w, dtype=dtype)
    at = torch.arange(n + more, dtype=torch.int32, device="cuda").expand(b, -1).contiguous()
    rq, rk = pages.rotate_prompt(rot, q, k, positions=at)
    outs, done = [], 0
    for size in (100, 1, 77, 52):
        sl = slice(done, done + size)
        before = pages.length.clone()
        pages.length += size
        pages.append(k[:, :, sl], v[:, :, sl], rotary=rot)
        keys, values = pages.read(done + size)
        outs.append(pages.attend_cross(rq[:, :, sl], keys, values, torch.full_like(before, size), pages.length, q_pos=before, mod=mod))
        done += size
    keys, values = pages.read(n)
    full = torch.full((b,), n, dtype=torch.int32, device="cuda")
    if not eight:
        assert torch.equal(keys, rk[:, :, :n]) and torch.equal(values, v[:, :, :n])
    want = pages.attend_prompt(rq[:, :, :n], keys, values, full, mod=mod).double()
    bound = 2 * tolerance(want, float(values.abs().max()), dtype, dtype == F32)  # each side within one of exact arithmetic
    if eight:  # a later chunk may have moved earlier codes of its page, each off by 2^-10 s then, s at most 1/224 of the largest entry. So a score moves by
        # scale * sum |q_c| * 2^-10 / 224 of the largest key, a weight relatively by as much (twice that, with the sum), a value by its own 2^-10 / 224.
        moved = 2.0 ** -10 / 224 * (2 * float(rq.float().abs().sum(-1).max()) / math.sqrt(d) * float(keys.abs().max()) + 1)
        bound = bound + moved * float(values.abs().max())
    assert bool(((torch.cat(outs, 2).double() - want).abs() <= bound).all())
    direct = HashEvictCache(b, h, g, d, 16, [n + more] * b, w, dtype=dtype)
    for c, kk, vv in ((cache, keys, values), (direct, rk[:, :, :n].contiguous(), v[:, :, :n].contiguous())):
        c.prefill_compress(rq[:, :, :n].contiguous(), kk, vv, full)
    if not eight:
        assert torch.equal(cache.codes, direct.codes) and torch.equal(cache.k_cache, direct.k_cache)
    for t in range(more):
        sl = slice(n + t, n + t + 1)
        pages.length += 1
        pages.append(k[:, :, sl], v[:, :, sl], rotary=rot)
        q_t, k_t = cache.rotate_step(rot, q[:, :, n + t].contiguous(), k[:, :, n + t].contiguous())
        assert torch.equal(k_t, rk[:, :, n + t])
        cache.decode_step(q_t, k_t, v[:, :, n + t].contiguous())
        a, c = pages.attend(q_t, mod), cache.attend_scored(q_t, mod)
        if not eight:  # the compressed cache holds everything: the same rows in another order
            assert bool(((a - c).abs() <= 4e-5 * float(v.abs().max())).all())
        every, _ = pages.read(n + t + 1)
        loss = cache.attention_loss(q_t, every)
        assert bool((loss.abs() <= 1e-5).all())


# (B, H, G, d, rows of each sequence, rows of the tensor, keys): at most 8 rows for a KV head, through the kernel of a new token's attention
FEW = [(3, 2, 4, 128, [1, 0, 1], 1, [1500, 40, 33]), (2, 1, 8, 64, [1, 1], 1, [2100, 700]), (2, 2, 1, 128, [8, 5], 8, [900, 31]), (1, 3, 2, 80, [3], 4, [1100]), (40, 2, 4, 64, [1] * 40, 1, [53 * i for i in range(40)]),
       (2, 2, 7, 120, [1, 1], 1, [640, 0]), (1, 1, 1, 8, [7], 7, [300])]


@pytest.mark.parametrize("opt", ["all keys", "all keys, cap", "all keys, first", "causal", "causal, cap + bias", "causal, window", "causal, ahead", "causal, behind"])
@pytest.mark.parametrize("b, h, g, d, q_lens, n, kv_lens", FEW)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_few_rows(b, h, g, d, q_lens, n, kv_lens, opt, layout):
    o = OPTIONS[opt]
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    m = max(kv_lens) + 5
    q, k, v = rows(gen, b, h * g, n, d, BF16, layout), rows(gen, b, h, m, d, BF16, layout) * 2, rows(gen, b, h, m, d, BF16, layout)
    kw = {}
    if o.get("causal"):
        kw["q_pos"] = torch.tensor([y - x + o.get("shift", 0) for x, y in zip(q_lens, kv_lens)], dtype=torch.int32, device="cuda")
    if "first" in o:
        kw["first_key"] = torch.randint(0, max(kv_lens) // 2 + 1, (b, n), generator=gen, device="cuda").sort(1).values.to(torch.int32)
    slopes = torch.exp2(-torch.arange(1, h * g + 1, device="cuda") * 8.0 / (h * g)) if o.get("slopes") else None
    mod = ScoreMod(scale=o.get("scale", 0.0), softcap=o.get("cap", 0.0), window=o.get("window", 0), slopes=slopes)
    for s in range(b):
        k[s, :, kv_lens[s]:], v[s, :, kv_lens[s]:] = math.nan, math.nan
    ql, kl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_lens, kv_lens))
    cache, out = make_cache(b, h, g, d, BF16), torch.full_like(q, 7.0)
    ws = torch.full((cache.cross_workspace(n, m).numel(),), 255, dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    cache.attend_cross(q, k, v, ql, kl, mod=mod, out=out, workspace=ws, **kw)
    check(out, q, k, v, q_lens, kv_lens, o, kw, slopes, g, n == 1 or "first" not in o and not o.get("causal"))
    again = torch.full_like(q, 7.0)
    cache.attend_cross(q, k, v, ql, kl, mod=mod, out=again, workspace=ws, **kw)
    assert torch.equal(out, again) and device_error_count() == 0


# rows of several query heads in one tile: 32 rows of four heads, 64 of two, groups that do not fill their last tile
PACKED = [(2, 2, 8, 128, BF16, [20, 29], [900, 300], "heads"), (1, 2, 7, 64, BF16, [5], [1400], "tokens"), (2, 1, 3, 80, BF16, [40, 61], [700, 500], "tokens"), (1, 3, 2, 128, BF16, [33], [600], "heads"),
          (2, 2, 5, 128, BF16, [61, 0], [129, 40], "heads"), (3, 1, 6, 64, BF16, [2, 29, 1], [0, 5, 2000], "heads")]


@pytest.mark.parametrize("opt", list(OPTIONS))
@pytest.mark.parametrize("shape", PACKED, ids=[f"{'x'.join(map(str, s[:4]))}-{max(s[5])}-{max(s[6])}" for s in PACKED])
@pytest.mark.parametrize("path", ["default", "whole"])
def test_rows_of_several_heads_in_a_tile(shape, opt, path, monkeypatch):
    test_attend_cross(shape, opt, path, monkeypatch)


@pytest.mark.parametrize("whole", [True, False])
def test_hidden_values_where_a_tile_holds_several_heads(whole):
    for opt in ("causal, window", "all keys, first"):
        test_hidden_infinities_and_nans_touch_nobody((1, 1, 4, 128, BF16, [30], [1500], "heads"), opt, whole)
