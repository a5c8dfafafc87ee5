"""The calls of sparse paged decoding and prefilling whose speed matters to a user of the library, as data, each with its plain form.

A layer of a serving step that attends a chosen part of a long history is a chain of operators over one paged KV cache:
``rope_kv_append`` (rotate Q and K by their positions, write K and V into the pages, keep the pages' bounds up to date),
``page_bounds_update`` (bounds of pages that were filled another way: a KV transfer), ``select_pages`` (a cheap score of every page
from its bounds, the best ones for each group of queries) and ``sparse_attn`` (attention over the selected pages).  Every pass goes
through the Python entry points with the buffers that a serving program keeps.  Where ``own`` is false ``run`` computes the same
from elementary torch operations.

What decides which pages are selected is held in whole numbers, and what leads up to those (rotated keys, page scales, bounds) is
computed in 64 bits and rounded once to each stored type, so that there is one right result, bit by bit.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

# Head geometry of the benchmark layers: (query heads, KV heads, head dimension, page size)
L8B = dict(Hq=32, Hkv=8, d=128, P=16)          # 8B-class layer
L32B = dict(Hq=64, Hkv=8, d=128, P=16)         # 32B-class layer
TP8 = dict(Hq=8, Hkv=1, d=128, P=32)           # one GPU's share of a 70B-class layer at TP = 8
SMALL = dict(Hq=8, Hkv=2, d=64, P=16)          # small model, head dimension 64
MID64 = dict(Hq=32, Hkv=8, d=64, P=64)         # head dimension 64 at the usual head count, large pages
GEOMETRIES = (L8B, L32B, TP8, SMALL, MID64)


def _case(name, op, geom, kv, *, dec=0, dc=(0, 0), pre=0, pc=(0, 0), pl=(0, 0), group=1, budget=0, first=1, last=2, rotary=0, interleaved=False,
          bounds=True, lengths=1):
    """dec decode rows with dc[0]..dc[1] cached tokens; pre rows with pc cached and pl new tokens (inclusive ranges; ``lengths``
    seeds the draw of the lengths inside them).  group, budget, first, last: queries per selection, pages per selection, and how many
    of those are the row's first and last pages whatever their score.  rotary: rotated elements of a head (0: all)."""
    c = dict(op=op, kv=kv, dec=dec, dc_lo=dc[0], dc_hi=dc[1], pre=pre, pc_lo=pc[0], pc_hi=pc[1], pl_lo=pl[0], pl_hi=pl[1], group=group,
             budget=budget, first=first, last=last, rotary=rotary or geom["d"], interleaved=interleaved, bounds=bounds, lengths=lengths, **geom)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one interactive session, one decode step: nothing but latency
        _case("rope_1_token", "rope", L8B, "bf16", dec=1, dc=(1533, 1533)),
        # a decode instance's batch at full load over the 8-bit cache
        _case("rope_96_tokens_8bit", "rope", L32B, "fp8", dec=96, dc=(2048, 16384)),
        # a batch of incremental prefills (configuration 2), half of each head rotated, neighbouring elements paired
        _case("rope_prefill_16_rows", "rope", L8B, "bf16", pre=16, pc=(1024, 8192), pl=(64, 1024), rotary=64, interleaved=True),
        # a decode worker has received the K/V of a short tool reply and of a batch of whole histories
        _case("bounds_1_reply", "bounds", L8B, "bf16", pre=1, pc=(2900, 2900), pl=(701, 701)),
        _case("bounds_16_histories", "bounds", L8B, "bf16", pre=16, pc=(0, 0), pl=(1024, 8192)),
        # long-context agent rounds (configuration 4): a decode step over a few long rows
        _case("select_4_long_rows", "select", TP8, "bf16", dec=4, dc=(36864, 69632), budget=64),
        # the decode instance at full load; 2 048 tokens are attended
        _case("select_96_rows", "select", L32B, "bf16", dec=96, dc=(2048, 16384), budget=128),
        # one incremental prefill over a long history, groups of 8 queries
        _case("select_prefill", "select", L8B, "bf16", pre=1, pc=(32771, 32771), pl=(509, 509), group=8, budget=128),
        # one session with a long history
        _case("sparse_1_row", "sparse", L8B, "bf16", dec=1, dc=(30011, 30011), budget=128),
        # the decode instance at full load
        _case("sparse_96_rows", "sparse", L32B, "bf16", dec=96, dc=(2048, 16384), budget=128),
        # the session trace's decode step over the 8-bit cache with large pages
        _case("sparse_25_rows_8bit", "sparse", MID64, "fp8", dec=25, dc=(4096, 32768), budget=32),
        # one incremental prefill over a long history, groups of 8 queries
        _case("sparse_prefill", "sparse", L8B, "bf16", pre=1, pc=(32771, 32771), pl=(509, 509), group=8, budget=128),
    ]


def _loguniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    a, b = sorted((_loguniform(rng, lo, hi), _loguniform(rng, lo, hi)))
    return a, b


def _seconds(case):
    """Rough cost of a pass, to compare cases with."""
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 1e15


def draw(rng):
    most = {op: max(_seconds(c) for c in listed() if c["op"] == op) for op in ("rope", "bounds", "select", "sparse")}
    while True:
        op = rng.choice(("rope", "bounds", "select", "select", "sparse", "sparse"))
        geom = rng.choice(GEOMETRIES)
        kind = "prefill" if op == "bounds" else rng.choice(("decode", "decode", "prefill", "mixed"))
        kw = dict(lengths=rng.randrange(1 << 20))
        if kind in ("decode", "mixed"):
            kw.update(dec=_loguniform(rng, 1, 128), dc=_span(rng, 256, 65536))
        if kind != "decode":
            pc = (0, 0) if rng.random() < 0.25 else _span(rng, 128, 65536)
            kw.update(pre=_loguniform(rng, 1, 4 if kind == "mixed" else 16), pc=pc, pl=_span(rng, 16, 1024 if op in ("select", "sparse") else 4096))
        if op == "rope":
            kw.update(rotary=rng.choice((geom["d"], geom["d"], geom["d"] // 2, geom["d"] // 4)), interleaved=rng.random() < 0.4,
                      bounds=rng.random() < 0.6)
        if op in ("select", "sparse"):
            most_group = 128 // (geom["Hq"] // geom["Hkv"])
            kw.update(group=1 if kind == "decode" else min(most_group, rng.choice((4, 8, 8, 16, 32))), first=rng.choice((0, 1, 1, 2)), last=rng.choice((1, 2, 4)))
            kw["budget"] = max(8, _loguniform(rng, 256, 4096) // geom["P"]) + rng.randrange(3)
        c = _case(None, op, geom, rng.choice(("bf16", "fp8")), **kw)
        C, L = _lengths(c)
        tokens = int(C.sum()) + int(L.sum())
        groups = int((-(-L // c["group"])).sum())
        gathered = groups * c["Hkv"] * c["budget"] * c["P"] * c["d"] if op == "sparse" else 0
        scored = len(C) * int((-(-L // c["group"])).max()) * int(C.max() + L.max()) // c["P"] * c["Hkv"] if op == "select" else 0
        padded = len(C) * int(C.max() + L.max()) // c["P"] * c["Hkv"] * 2 * c["d"] if op == "select" else 0
        if _seconds(c) <= most[op] and tokens * c["Hkv"] * c["d"] <= 3 << 30 and gathered <= 1 << 30 and scored <= 1 << 28 and padded <= 1 << 30:
            return c


def _lengths(case):
    """Cached and new tokens of every row; prefill rows are spread among the decode rows."""
    g = np.random.default_rng(case["lengths"])
    Cd = g.integers(case["dc_lo"], case["dc_hi"], size=case["dec"], endpoint=True)
    Cp = g.integers(case["pc_lo"], case["pc_hi"], size=case["pre"], endpoint=True)
    Lp = g.integers(case["pl_lo"], case["pl_hi"], size=case["pre"], endpoint=True)
    n = case["dec"] + case["pre"]
    C, L = np.empty(n, np.int32), np.ones(n, np.int32)
    is_pre = np.zeros(n, bool)
    if case["pre"]:
        is_pre[np.linspace(0, n - 1, case["pre"]).astype(np.int64)] = True
    C[is_pre], L[is_pre], C[~is_pre] = Cp, Lp, Cd
    return C, L


# ---- inputs ----------------------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    """The inputs, the same ones for either form, and for the framework's calls the descriptors and the workspace that go with them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    Hq, Hkv, d, P, op = case["Hq"], case["Hkv"], case["d"], case["P"], case["op"]
    fp8 = case["kv"] == "fp8"
    C, L = _lengths(case)
    pages_of = -(-(C.astype(np.int64) + L) // P)
    used = int(pages_of.sum())
    pages = math.ceil(1.1 * used) + 1
    perm = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32).cpu().numpy()
    bt = np.full((len(C), int(pages_of.max())), -1, np.int32)
    o = 0
    for r, k in enumerate(pages_of):
        bt[r, :k] = perm[o:o + k]
        o += int(k)
    s = dict(case=dict(case), C=C, L=L, bt=torch.from_numpy(bt).cuda(), ctx=torch.from_numpy(C).cuda().long(), incr=torch.from_numpy(L).cuda().long())
    n = int(L.sum())

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    def bounds():
        # the bounds of pages of P keys that are about normal: some 2 above and below zero, in units of the page's scale
        codes = torch.empty((pages, Hkv, 2, d), device="cuda", dtype=torch.int8)
        codes[:, :, 0] = (62 + 15 * torch.randn((pages, Hkv, d), generator=gen, device="cuda", dtype=torch.float16)).clamp(-127, 127).to(torch.int8)
        codes[:, :, 1] = (-62 + 15 * torch.randn((pages, Hkv, d), generator=gen, device="cuda", dtype=torch.float16)).clamp(-127, 127).to(torch.int8)
        return SimpleNamespace(codes=codes, scale=torch.exp2(torch.randint(-6, -4, (pages, Hkv), generator=gen, device="cuda").float()))

    k_scale = v_scale = None
    if op == "select":
        # the selection reads bounds and queries; the pools are there, but no pass touches them
        k_pool, v_pool = (torch.empty((pages, Hkv, P, d), device="cuda", dtype=torch.uint8 if fp8 else torch.bfloat16) for _ in range(2))
        if fp8:
            k_scale, v_scale = (torch.ones((pages, Hkv), device="cuda") for _ in range(2))
    elif fp8:
        exps = torch.randint(-7, -5, (2, pages, Hkv), generator=gen, device="cuda").float()
        k_scale, v_scale = torch.exp2(exps[0]), torch.exp2(exps[1])
        k_pool, v_pool = ((normal(pages, Hkv, P, d) / sc[:, :, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                          for sc in (k_scale, v_scale))
    else:
        k_pool, v_pool = normal(pages, Hkv, P, d), normal(pages, Hkv, P, d)
    s["cache"] = SimpleNamespace(k_pool=k_pool, v_pool=v_pool, k_scale=k_scale, v_scale=v_scale, kv_dtype=int(fp8), softmax_scale=1.0 / math.sqrt(d))
    s["bounds"] = bounds() if op in ("bounds", "select") or op == "rope" and case["bounds"] else None
    groups = int((-(-L // case["group"])).sum())
    if op == "rope":
        # Q, K and V of a token lie next to each other, as one projection writes them
        s["qkv"] = normal(n, (Hq + 2 * Hkv) * d)
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, case["rotary"], 2, device="cuda", dtype=torch.float64) / case["rotary"])).float()
        s["q_out"] = torch.empty((n, Hq, d), device="cuda", dtype=torch.bfloat16)
    elif op != "bounds":
        s["q"] = normal(n, Hq, d)
    if op == "select":
        s["selected"] = torch.empty((groups, Hkv, case["budget"]), device="cuda", dtype=torch.int32)
    elif op == "sparse":
        # what a selection finds: pages that matter to the whole row, and pages that matter to one group of queries
        req, lp_first, lp_last = _groups(s["ctx"], s["incr"], groups, case["group"], P)[:3]
        score = torch.randn((len(C), Hkv, bt.shape[1]), generator=gen, device="cuda")[req]
        score += torch.randn((groups, Hkv, bt.shape[1]), generator=gen, device="cuda")
        s["selected"] = _choose(score, lp_first, lp_last, case)
        s["out"] = torch.empty_like(s["q"])
    if own:
        import paper_2602_14516_amd as A
        s["A"] = A
        s["handle"] = A.KVCache(Hq, Hkv, d, P, k_pool, v_pool, s["cache"].softmax_scale, k_scale, v_scale, s["cache"].kv_dtype)
        s["page_bounds"] = A.PageBounds(s["bounds"].codes, s["bounds"].scale) if s["bounds"] is not None else None
        if op == "rope":
            s["rope"] = A.Rope(s["inv_freq"], interleaved=case["interleaved"])
        elif op == "select":
            ws = A.select_pages_workspace_bytes(s["handle"], C, L, bt.shape[1], case["budget"], first_pages=case["first"], last_pages=case["last"],
                                                group_tokens=case["group"])
            s["workspace"] = torch.empty(max(ws, 256), device="cuda", dtype=torch.uint8)
        elif op == "sparse":
            ws = A.sparse_attn_workspace_bytes(s["handle"], C, L, bt.shape[1], case["budget"], group_tokens=case["group"])
            s["workspace"] = torch.empty(max(ws, 256), device="cuda", dtype=torch.uint8)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------------


def run(s):
    op, cache, case = s["case"]["op"], s["cache"], s["case"]
    if own:
        A, handle = s["A"], s["handle"]
        if op == "rope":
            q, k, v = _split(s)
            A.rope_kv_append(handle, s["C"], s["L"], s["bt"], s["rope"], q, k, v, q_out=s["q_out"], bounds=s["page_bounds"])
        elif op == "bounds":
            A.page_bounds_update(handle, s["C"], s["L"], s["bt"], s["page_bounds"])
        elif op == "select":
            A.select_pages(handle, s["C"], s["L"], s["bt"], s["page_bounds"], s["q"], case["budget"], first_pages=case["first"],
                           last_pages=case["last"], group_tokens=case["group"], out=s["selected"], workspace=s["workspace"])
        else:
            A.sparse_attn(handle, s["C"], s["L"], s["bt"], s["selected"], s["q"], group_tokens=case["group"], out=s["out"], workspace=s["workspace"])
    else:
        {"rope": _plain_rope, "bounds": _plain_bounds, "select": _plain_select, "sparse": _plain_sparse}[op](s)
    if op == "rope":
        # 8-bit pages as the numbers of their type; their scales, and the bounds', beside them
        pools = [t.view(torch.float8_e4m3fn) if t.dtype == torch.uint8 else t for t in (cache.k_pool, cache.v_pool)]
        more = [cache.k_scale, cache.v_scale] if cache.kv_dtype == 1 else []
        return [s["q_out"], *pools, *more] + ([s["bounds"].codes, s["bounds"].scale] if s["bounds"] is not None else [])
    return {"bounds": lambda: [s["bounds"].codes, s["bounds"].scale], "select": lambda: [s["selected"]], "sparse": lambda: [s["out"]]}[op]()


def _split(s):
    """Q, K and V [tokens, heads, d] as views of the projection's rows."""
    c = s["case"]
    x = s["qkv"].view(len(s["qkv"]), c["Hq"] + 2 * c["Hkv"], c["d"])
    return x[:, :c["Hq"]], x[:, c["Hq"]:c["Hq"] + c["Hkv"]], x[:, c["Hq"] + c["Hkv"]:]


def _tokens(ctx, incr, n):
    """Row and position of every new token."""
    req = torch.repeat_interleave(torch.arange(len(ctx), device=ctx.device), incr, output_size=n)
    return req, ctx[req] + torch.arange(n, device=ctx.device) - (incr.cumsum(0) - incr)[req]


def _groups(ctx, incr, groups, g, P):
    """Of every group of g new tokens: row, page of its first and of its last token, packed index of its first token, tokens, ordinal in
    its row."""
    per = (incr + g - 1) // g
    req = torch.repeat_interleave(torch.arange(len(ctx), device=ctx.device), per, output_size=groups)
    at = torch.arange(groups, device=ctx.device) - (per.cumsum(0) - per)[req]
    count = torch.minimum(incr[req] - at * g, torch.tensor(g, device=ctx.device))
    first = ctx[req] + at * g
    return req, first // P, (first + count - 1) // P, (incr.cumsum(0) - incr)[req] + at * g, count, at


def _choose(score, lp_first, lp_last, case):
    """The best `budget` pages of score [groups, Hkv, pages] (ties: the lowest index), ascending, -1 behind; the first pages and those from
    the group's first token's window to its last token's page always."""
    j = torch.arange(score.shape[2], device=score.device)
    forced = (j < case["first"]) | (j >= (lp_first - (case["last"] - 1))[:, None])
    there = j <= lp_last[:, None]
    score = torch.where((forced & there)[:, None], torch.tensor(math.inf, device=score.device, dtype=score.dtype), score)
    score = torch.where(there[:, None], score, torch.tensor(-math.inf, device=score.device, dtype=score.dtype))
    best, at = torch.sort(score, dim=2, descending=True, stable=True)
    k = min(case["budget"], score.shape[2])
    big = score.shape[2]
    at = torch.where(best[:, :, :k] == -math.inf, big, at[:, :, :k]).sort(dim=2).values
    out = torch.full((*score.shape[:2], case["budget"]), -1, device=score.device, dtype=torch.int32)
    out[:, :, :k] = torch.where(at == big, -1, at)
    return out


def _rotate(x, cos, sin, interleaved):
    """x [tokens, heads, d] in cos's type; cos, sin [tokens, rotary / 2]."""
    h = cos.shape[1]
    c, s_ = cos[:, None], sin[:, None]
    a, b = (x[:, :, 0:2 * h:2], x[:, :, 1:2 * h:2]) if interleaved else (x[:, :, :h], x[:, :, h:2 * h])
    y = torch.stack((a * c - b * s_, b * c + a * s_), dim=3 if interleaved else 2).flatten(2)
    return torch.cat((y, x[:, :, 2 * h:]), dim=2)


def _pages_touched(s, n):
    """Of every page that new tokens fall into: physical page, its first position, row; of every token: which of those its page is, and
    its slot."""
    ctx, incr, P = s["ctx"], s["incr"], s["case"]["P"]
    per = torch.where(incr > 0, (ctx + incr - 1) // P - ctx // P + 1, 0)
    count = int(((s["C"].astype(np.int64) + s["L"] - 1) // P - s["C"] // P + 1)[s["L"] > 0].sum())
    before = per.cumsum(0) - per
    row = torch.repeat_interleave(torch.arange(len(ctx), device=ctx.device), per, output_size=count)
    lp = ctx[row] // P + torch.arange(count, device=ctx.device) - before[row]
    req, pos = _tokens(ctx, incr, n)
    return s["bt"][row, lp].long(), lp * P, row, before[req] + pos // P - ctx[req] // P, pos % P


def _exponent(amax, most, lo, hi):
    """The smallest e with amax <= most * 2^e, within lo..hi."""
    m, e = torch.frexp(amax.double() / most)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(amax > 0, e, lo).clamp(lo, hi)


def _stored_keys(cache, page):
    """Keys of whole pages as the cache holds them, [pages, Hkv, P, d] in 32 bits."""
    if cache.kv_dtype == 1:
        return cache.k_pool[page].view(torch.float8_e4m3fn).float() * cache.k_scale[page][:, :, None, None]
    return cache.k_pool[page].float()


def _plain_bounds_of(s, page, first, row):
    P = s["case"]["P"]
    k = _stored_keys(s["cache"], page)
    there = (first[:, None] + torch.arange(P, device=page.device) < (s["ctx"] + s["incr"])[row][:, None])[:, None, :, None]
    hi, lo = k.masked_fill(~there, -math.inf).amax(2), k.masked_fill(~there, math.inf).amin(2)
    e = _exponent(torch.maximum(hi.abs(), lo.abs()).amax(2), 127.0, -40, 96)
    inv = torch.exp2(-e.double())[:, :, None]
    s["bounds"].codes[page] = torch.stack(((hi * inv).ceil(), (lo * inv).floor()), 2).clamp(-127, 127).to(torch.int8)
    s["bounds"].scale[page] = torch.exp2(e.float())


def _plain_bounds(s):
    page, first, row = _pages_touched(s, int(s["L"].sum()))[:3]
    _plain_bounds_of(s, page, first, row)


def _plain_rope(s):
    cache, case = s["cache"], s["case"]
    n, P = len(s["qkv"]), case["P"]
    q, k, v = _split(s)
    req, pos = _tokens(s["ctx"], s["incr"], n)
    angle = pos.double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos(), angle.sin()
    s["q_out"].copy_(_rotate(q.float(), cos.float(), sin.float(), case["interleaved"]))
    k = _rotate(k.double(), cos, sin, case["interleaved"]).float().to(torch.bfloat16)     # keys decide codes and page choices: 64 bits
    page, first, row, of, slot = _pages_touched(s, n)
    if cache.kv_dtype == 1:
        _quantise(s, k, cache.k_pool, cache.k_scale, page, first, row, of, slot)
        _quantise(s, v, cache.v_pool, cache.v_scale, page, first, row, of, slot)
    else:
        cache.k_pool[page[of], :, slot] = k
        cache.v_pool[page[of], :, slot] = v
    if s["bounds"] is not None:
        _plain_bounds_of(s, page, first, row)


def _quantise(s, x, pool, scale, page, first, row, of, slot):
    """x [tokens, Hkv, d] into 8-bit pages: a page's exponent never falls, and its old codes follow when it rises."""
    amax = torch.zeros((len(page), x.shape[1]), device=x.device).index_reduce(0, of, x.float().abs().amax(2), "amax")
    e = _exponent(amax, 448.0, -40, 119)
    held = s["ctx"][row] - first                                                           # slots that already hold tokens
    e = torch.where((held > 0)[:, None], torch.maximum(e, torch.frexp(scale[page])[1] - 1), e)
    codes = pool[page].view(torch.float8_e4m3fn).float() * (scale[page].double() * torch.exp2(-e.double())).float()[:, :, None, None]
    codes = codes.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    old = (torch.arange(pool.shape[2], device=x.device) < held[:, None])[:, None, :, None]
    pool[page] = torch.where(old, codes, pool[page])
    inv = torch.exp2(-e.double())[of][:, :, None]
    pool[page[of], :, slot] = (x.double() * inv).float().to(torch.float8_e4m3fn).view(torch.uint8)
    scale[page] = torch.exp2(e.float())


def _plain_select(s):
    case, b = s["case"], s["bounds"]
    g, Hkv, d, R = case["group"], case["Hkv"], case["d"], len(s["C"])
    groups, most = s["selected"].shape[0], int((-(-s["L"] // g)).max())
    req, lp_first, lp_last, tok0, count, at = _groups(s["ctx"], s["incr"], groups, g, case["P"])
    tok = tok0[:, None] + torch.arange(g, device=req.device)
    in_group = torch.arange(g, device=req.device) < count[:, None]
    q = s["q"][tok.clamp(max=len(s["q"]) - 1)].float().view(groups, g, Hkv, -1, d)
    q = torch.where(in_group[:, :, None, None, None], q, 0.0)
    e = _exponent(q.abs().amax(dim=(1, 3, 4)), 127.0, -140, 127)
    c = (q * torch.exp2(-e.double())[:, None, :, None, None]).round()                      # 64 bits, ties to even
    c = torch.cat((c.clamp(min=0).sum((1, 3)), c.clamp(max=0).sum((1, 3))), 2)             # [groups, Hkv, 2 d], whole numbers
    rows = torch.zeros((R, most, Hkv, 2 * d), device=c.device, dtype=torch.float64)
    rows[req, at] = c
    page = s["bt"].clamp(min=0).long()                                                     # [R, pages]
    codes = b.codes[page].flatten(3).double().permute(0, 2, 3, 1)                          # [R, Hkv, 2 d, pages]
    total = torch.matmul(rows.transpose(1, 2), codes)                                      # whole numbers below 2^31: exact in 64 bits
    score = total.float() * b.scale[page].permute(0, 2, 1)[:, :, None]
    s["selected"].copy_(_choose(score.transpose(1, 2)[req, at], lp_first, lp_last, case))


def _plain_sparse(s):
    case, cache, sel = s["case"], s["cache"], s["selected"]
    g, Hkv, d, P = case["group"], case["Hkv"], case["d"], case["P"]
    groups, n = sel.shape[0], len(s["q"])
    req, _, lp_last, tok0, count, at = _groups(s["ctx"], s["incr"], groups, g, P)
    tok = (tok0[:, None] + torch.arange(g, device=req.device)).clamp(max=n - 1)
    in_group = torch.arange(g, device=req.device) < count[:, None]
    listed_ = (sel >= 0) & (sel <= lp_last[:, None, None])
    page = s["bt"][req[:, None, None], sel.clamp(min=0)].clamp(min=0).long()               # [groups, Hkv, budget]
    head = torch.arange(Hkv, device=req.device)[None, :, None]

    def rows(pool, scale):
        x = pool[page, head]                                                               # [groups, Hkv, budget, P, d]
        x = x.view(torch.float8_e4m3fn).float() * scale[page, head][..., None, None] if cache.kv_dtype == 1 else x.float()
        return x.flatten(2, 3)

    pos = (sel * P)[..., None] + torch.arange(P, device=req.device)                        # [groups, Hkv, budget, P]
    pos = torch.where(listed_[..., None], pos, 1 << 30).flatten(2)
    seen = pos[:, :, None] <= (s["ctx"][req] + at * g)[:, None, None, None] + torch.arange(g, device=req.device)[:, None]   # [groups, Hkv, g, keys]
    q = s["q"][tok].float().view(groups, g, Hkv, -1, d).transpose(1, 2).flatten(2, 3)      # [groups, Hkv, g G, d]
    G = q.shape[2] // g
    logits = torch.matmul(q, rows(cache.k_pool, cache.k_scale).transpose(2, 3)) * cache.softmax_scale
    logits = logits.masked_fill(~seen.repeat_interleave(G, dim=2), -math.inf)
    p = (logits - logits.amax(3, keepdim=True).clamp(min=-1e30)).exp()
    total = p.sum(3, keepdim=True)
    v = torch.where(seen.any(2)[..., None], rows(cache.v_pool, cache.v_scale), 0.0)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    o = o.view(groups, Hkv, g, G, d).transpose(1, 2).flatten(2, 3)                         # [groups, g, Hq, d]
    s["out"][tok[in_group]] = o[in_group].to(torch.bfloat16)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------------


def exact(case, seed):
    """Row by row and page by page in 64 bits: what run() returns for these inputs."""
    s = prepare(case, seed)
    cache, op, P, d, Hkv, Hq = s["cache"], case["op"], case["P"], case["d"], case["Hkv"], case["Hq"]
    G, g, fp8 = Hq // Hkv, case["group"], case["kv"] == "fp8"
    bt = s["bt"].cpu().numpy()

    def e4m3(x):
        return x.to(torch.float32).to(torch.float8_e4m3fn)                                 # (a 64-bit value of few bits is exact in 32)

    def smallest(amax, most, lo, hi):
        e = torch.log2((amax / most).clamp(min=1e-300)).ceil().clamp(lo, hi)
        e = torch.where(amax > most * torch.exp2(e), e + 1, e)
        return torch.where(amax <= most * torch.exp2(e - 1), e - 1, e).clamp(lo, hi)

    def set_bounds(r, lp, end):
        page = int(bt[r, lp])
        k = cache.k_pool[page].view(torch.float8_e4m3fn).double() * cache.k_scale[page].double()[:, None, None] if fp8 else cache.k_pool[page].double()
        k = k[:, :end - lp * P]
        hi, lo = k.max(1).values, k.min(1).values
        e = smallest(k.abs().amax((1, 2)), 127.0, -40, 40)
        s["bounds"].codes[page, :, 0] = torch.ceil(hi / torch.exp2(e)[:, None]).to(torch.int8)
        s["bounds"].codes[page, :, 1] = torch.floor(lo / torch.exp2(e)[:, None]).to(torch.int8)
        s["bounds"].scale[page] = torch.exp2(e).float()

    if op in ("rope", "bounds"):
        pages = sum(int(-(-(c + n) // P) - c // P) for c, n in zip(s["C"], s["L"]))
        if pages > 15000:                                                                  # a page at a time: about 20 s
            return None
    if op == "bounds":
        for r, (c, n) in enumerate(zip(s["C"].tolist(), s["L"].tolist())):
            for lp in range(c // P, (c + n - 1) // P + 1):
                set_bounds(r, lp, min(c + n, (lp + 1) * P))
        return [s["bounds"].codes, s["bounds"].scale]
    if op == "rope":
        x = s["qkv"].double().view(-1, Hq + 2 * Hkv, d)
        h = case["rotary"] // 2
        row0, q_rows = 0, []
        for r, (c, n) in enumerate(zip(s["C"].tolist(), s["L"].tolist())):
            xr = x[row0:row0 + n]
            row0 += n
            at = torch.arange(c, c + n, device="cuda", dtype=torch.float64)
            turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), at[:, None] * s["inv_freq"].double())[:, None]
            qk = xr[:, :Hq + Hkv]
            if case["interleaved"]:
                z = torch.view_as_complex(qk[..., :2 * h].reshape(n, Hq + Hkv, h, 2)) * turn
                y = torch.view_as_real(z).reshape(n, Hq + Hkv, 2 * h)
            else:
                z = torch.complex(qk[..., :h].contiguous(), qk[..., h:2 * h].contiguous()) * turn
                y = torch.cat((z.real, z.imag), 2)
            y = torch.cat((y, qk[..., 2 * h:]), 2)
            q_rows.append(y[:, :Hq])
            kv = ((cache.k_pool, cache.k_scale, y[:, Hq:].float().to(torch.bfloat16)), (cache.v_pool, cache.v_scale, s["qkv"].view(-1, Hq + 2 * Hkv, d)[row0 - n:row0, Hq + Hkv:]))
            for lp in range(c // P, (c + n - 1) // P + 1):
                page, t0, t1 = int(bt[r, lp]), max(c, lp * P), min(c + n, (lp + 1) * P)
                for pool, scale, rows in kv:
                    new = rows[t0 - c:t1 - c].transpose(0, 1)                              # [Hkv, tokens, d]
                    if not fp8:
                        pool[page, :, t0 - lp * P:t1 - lp * P] = new
                        continue
                    e = smallest(new.double().abs().amax((1, 2)), 448.0, -40, 40)
                    if t0 > lp * P:
                        was = torch.log2(scale[page].double())
                        e = torch.maximum(e, was)
                        old = pool[page, :, :t0 - lp * P].view(torch.float8_e4m3fn).double() * torch.exp2(was - e)[:, None, None]
                        pool[page, :, :t0 - lp * P] = e4m3(old).view(torch.uint8)
                    pool[page, :, t0 - lp * P:t1 - lp * P] = e4m3(new.double() / torch.exp2(e)[:, None, None]).view(torch.uint8)
                    scale[page] = torch.exp2(e).float()
                if case["bounds"]:
                    set_bounds(r, lp, t1)
        pools = [t.view(torch.float8_e4m3fn) if fp8 else t for t in (cache.k_pool, cache.v_pool)]
        return [torch.cat(q_rows), *pools] + ([cache.k_scale, cache.v_scale] if fp8 else []) + ([s["bounds"].codes, s["bounds"].scale] if case["bounds"] else [])
    row0, out, chosen = 0, [], []
    at = 0
    for r, (c, n) in enumerate(zip(s["C"].tolist(), s["L"].tolist())):
        q_row = s["q"][row0:row0 + n].double().view(n, Hkv, G, d)
        row0 += n
        pages = torch.from_numpy(bt[r, :-(-(c + n) // P)]).cuda().long()
        if op == "select":
            hi, lo = (s["bounds"].codes[pages][:, :, i].permute(1, 2, 0).long() for i in (0, 1))       # [Hkv, d, pages]
        else:
            k_row, v_row = (pool[pages].view(torch.float8_e4m3fn).double() * sc[pages].double()[:, :, None, None] if fp8 else pool[pages]
                            for pool, sc in ((cache.k_pool, cache.k_scale), (cache.v_pool, cache.v_scale)))
        for i in range(0, n, g):
            q = q_row[i:i + g].transpose(0, 1)                                             # [Hkv, tokens, G, d]
            m = q.shape[1]
            if op == "select":
                lp0, lp1 = (c + i) // P, (c + i + m - 1) // P
                e = smallest(q.abs().amax((1, 2, 3)), 127.0, -40, 40)
                code = torch.round(q / torch.exp2(e)[:, None, None, None])
                pos, neg = (torch.clamp(code, **kw).sum((1, 2)) for kw in ({"min": 0}, {"max": 0}))
                total = (pos[:, :, None] * hi.double() + neg[:, :, None] * lo.double()).sum(1)
                score = total.float() * s["bounds"].scale[pages].t()                       # [Hkv, pages]
                always = [j for j in range(lp1 + 1) if j < case["first"] or j > lp0 - case["last"]]
                rest = [j for j in range(lp1 + 1) if case["first"] <= j <= lp0 - case["last"]]
                left = min(case["budget"] - len(always), len(rest))
                row = np.full((Hkv, case["budget"]), -1, np.int32)
                sc = score.cpu().numpy()
                for hd in range(Hkv):
                    best = [rest[j] for j in np.argsort(-sc[hd, rest], kind="stable")[:left]] if left > 0 else []
                    row[hd, :len(always) + len(best)] = sorted(always + best)
                chosen.append(torch.from_numpy(row).cuda())
                continue
            o = torch.zeros((m, Hkv, G, d), device="cuda", dtype=torch.float64)
            sel = s["selected"][at].long()                                                 # [Hkv, budget]
            at += 1
            use = sel.clamp(min=0)
            heads = torch.arange(Hkv, device="cuda")[:, None]
            k = k_row[use, heads].double().flatten(1, 2)                                   # [Hkv, keys, d]
            v = v_row[use, heads].double().flatten(1, 2)
            pos = torch.where(sel >= 0, sel * P, 1 << 40)[:, :, None] + torch.arange(P, device="cuda")
            see = pos.flatten(1)[:, None, None] <= torch.arange(c + i, c + i + m, device="cuda")[:, None, None]
            w = torch.matmul(q, k.transpose(1, 2)[:, None]) * cache.softmax_scale
            w = torch.softmax(w.masked_fill(~see, -math.inf), 3)
            o += torch.matmul(w, torch.where(see.any((1, 2))[..., None], v, 0.0)[:, None]).transpose(0, 1)
            out.append(o.reshape(m, Hq, d))
    return [torch.stack(chosen)] if op == "select" else [torch.cat(out)]


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------


def work(case):
    C, L = (x.astype(np.int64) for x in _lengths(case))
    Hq, Hkv, d, P, op, g = case["Hq"], case["Hkv"], case["d"], case["P"], case["op"], case["group"]
    b = 1 if case["kv"] == "fp8" else 2
    T = C + L
    first = C // P
    pages = (T - 1) // P - first + 1                                # that new tokens fall into
    groups = -(-L // g)
    if op == "rope":
        byt = L * ((Hq + 2 * Hkv) * d * 2 + Hq * d * 2 + 2 * Hkv * d * b) + 4 * pages
        if b == 1:
            byt = byt + pages * Hkv * 2 * 4
        if case["bounds"]:                                          # the cached keys that share a page with new ones are read
            byt = byt + pages * Hkv * (2 * d + 4) + (C - first * P) * Hkv * d * b
        return {"bytes": int(byt.sum()) + case["rotary"] * 2, "flops": int((L * (Hq + Hkv) * case["rotary"] * 3).sum())}
    if op == "bounds":
        byt = (T - first * P) * Hkv * d * b + pages * (Hkv * (2 * d + 4 + (4 if b == 1 else 0)) + 4)
        return {"bytes": int(byt.sum()), "flops": int(((T - first * P) * Hkv * d * 2).sum())}
    if op == "select":
        row_pages = np.maximum(0, (T - 1) // P + 1 - case["first"] - case["last"])
        byt = row_pages * (Hkv * (2 * d + 4) + 4) + L * Hq * d * 2 + groups * Hkv * case["budget"] * 4
        return {"bytes": int(byt.sum()), "flops": int((groups * row_pages * Hkv * 4 * d).sum())}
    row_pages = (T - 1) // P + 1
    keys = np.minimum(case["budget"], row_pages) * P
    read = np.minimum(groups * np.minimum(case["budget"], row_pages), row_pages)   # every page of a row at most once for each KV head
    byt = read * Hkv * (P * d * b * 2 + (8 if b == 1 else 0)) + L * Hq * d * 2 * 2 + groups * Hkv * case["budget"] * 4
    return {"bytes": int(byt.sum()), "flops": int((4 * d * Hq * L * keys).sum())}
