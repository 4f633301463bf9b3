"""The paged cache's operators as they are timed: rotary positions, the append into pages, attention of one new
token over pages, and eviction by accumulated attention weight.

A case is one pass of an operator.  With `own` false a pass is the operator's definition in elementary torch
operations, in 32 bits (angles in 64); with `own` true it is the package's call.  exact() restates the
definitions in 64 bits, apart from both.
"""
import math
import random

import numpy as np
import torch

own = False

_DTYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _named(name, c):
    return dict(c, name=name) if name else c


def _rope(name, tokens, heads, dim, rotary, dtype, interleaved=False, scaling="none", far=131072, backward=False,
          fused=False):
    return _named(name, dict(kind="rope", tokens=tokens, heads=heads, dim=dim, rotary=rotary, dtype=dtype,
                             interleaved=interleaved, scaling=scaling, far=far, backward=backward, fused=fused))


def _append(name, seqs, longest, new, heads, dim, page, store, group_s=16, rope=True, heads_first=False):
    return _named(name, dict(kind="append", seqs=seqs, longest=longest, new=new, heads=heads, dim=dim, page=page,
                             store=store, group_s=group_s, rope=rope, heads_first=heads_first))


def _attend(name, seqs, q_heads, kv_heads, dim, longest, ragged, page, store, group_s=16, window=0, out="float16",
            weights=False, heads_first=False):
    return _named(name, dict(kind="attend", seqs=seqs, q_heads=q_heads, kv_heads=kv_heads, dim=dim, longest=longest,
                             ragged=ragged, page=page, store=store, group_s=group_s, window=window, out=out,
                             weights=weights, heads_first=heads_first))


def _evict(name, seqs, kv_heads, dim, longest, ragged, budget, recent, sinks, page, store, heads_first=False):
    return _named(name, dict(kind="evict", seqs=seqs, kv_heads=kv_heads, dim=dim, longest=longest, ragged=ragged,
                             budget=budget, recent=recent, sinks=sinks, page=page, store=store,
                             heads_first=heads_first))


def listed():
    return [
        # the queries of one decode step, 16 sequences at positions of a long context: latency alone
        _rope("rope_step", 16, 32, 128, 128, "float16", scaling="llama3"),
        # the queries of a long prompt, rotated inside the fused qkv projection's output
        _rope("rope_prompt", 8192, 32, 128, 128, "bfloat16", scaling="yarn", fused=True),
        # pairs side by side, half of an odd head rotated, an odd token count, 32-bit gradients
        _rope("rope_partial_grad", 4001, 20, 96, 64, "float32", interleaved=True, backward=True),
        # one new token for each of 64 sequences, key rotated on its way into its page
        _append("append_step", 64, 2048, 1, 8, 128, 16, "bfloat16"),
        # prompts encoded into 4-bit pages and read back for the prompt's own attention
        _append("append_prompt_lzs", 8, 2048, 2048, 8, 128, 64, "lzs"),
        # one sequence, a short odd context, every query head with its own keys: latency
        _attend("attn_one_777", 1, 40, 40, 128, 777, False, 16, "float16"),
        # a batch of sequences of all lengths, four query heads to a key head, 16-bit pages
        _attend("attn_batch", 32, 32, 8, 128, 8192, True, 16, "bfloat16", out="bfloat16"),
        # a few long contexts in 4-bit pages, eight query heads to a key head
        _attend("attn_long_lzs", 8, 64, 8, 128, 65536, True, 64, "lzs"),
        # 4-bit pages whose attention weights are accumulated for a later eviction
        _attend("attn_weights_lzs", 16, 32, 8, 128, 4096, True, 32, "lzs", group_s=8, weights=True),
        # wide heads that see a window of the last tokens only
        _attend("attn_window_256", 24, 16, 8, 256, 16384, True, 32, "float16", window=4096, heads_first=True),
        # a budget just passed: a few rows go, all of the rest close up
        _evict("evict_step", 4, 8, 128, 2112, False, 2048, 256, 4, 16, "float16"),
        # a batch of long contexts cut to a quarter
        _evict("evict_long", 16, 8, 128, 16384, True, 4096, 512, 4, 64, "bfloat16", heads_first=True),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    what = rng.choice(["rope", "append"] + ["attend"] * 4 + ["evict"])
    page = rng.choice([8, 16, 32, 64, 128])
    first = rng.random() < 0.5
    if what == "rope":
        dim = rng.choice([64, 80, 96, 128, 192, 256])
        heads = _log(rng, 1, 64)
        tokens = _log(rng, 1, 8192 * 32 * 128 // (dim * heads))
        dtype = rng.choice(["float16", "bfloat16", "float32"])
        if dtype == "float32":
            tokens = max(1, tokens // 2)
        return _rope(None, min(tokens, 65536), heads, dim, rng.choice([dim, dim, dim // 2]), dtype,
                     rng.random() < 0.5, rng.choice(["none", "linear", "yarn", "llama3"]),
                     _log(rng, 4096, 1 << 20), rng.random() < 0.3, rng.random() < 0.3)
    dim = rng.choice([64, 128, 128, 192, 256])
    store = rng.choice(["float16", "bfloat16", "lzs", "lzs"])
    gs = rng.choice([8, 16, 16, 32, 64])
    kv = _log(rng, 1, 16)
    if what == "append":
        new = _log(rng, 1, 1024)
        seqs = _log(rng, 1, max(1, min(64, 16384 * 8 * 128 // (new * kv * dim))))
        return _append(None, seqs, new + rng.randrange(1024), new, kv, dim, page, store, gs, rng.random() < 0.7, first)
    if what == "attend":
        group = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
        seqs = _log(rng, 1, 64)
        most = 4 * 65536 * 8 * 128 // (seqs * kv * dim * (1 if store == "lzs" else 4))
        longest = _log(rng, 1, min(65536, max(1, most)))
        window = rng.choice([0, 0, 0, rng.randrange(1, longest + 64)])
        return _attend(None, seqs, kv * group, kv, dim, longest, rng.random() < 0.7, page, store, gs, window,
                       rng.choice(["float16", "bfloat16", "float32"]), rng.random() < 0.3, first)
    if store == "lzs":
        store = "float16"
    seqs = _log(rng, 1, 16)
    longest = _log(rng, 16, min(16384, max(16, 8 * 16384 * 8 * 128 // (seqs * kv * dim))))
    budget = max(8, int(longest * rng.uniform(0.2, 1.05)))
    recent = rng.randrange(0, budget // 2)
    return _evict(None, seqs, kv, dim, longest, rng.random() < 0.7, budget, recent, rng.randrange(0, 5), page, store,
                  first)


def _lens(case):
    """The sequences' lengths: of the case alone.  Ragged ones spread over the whole range (one is the longest,
    and of eight or more one is empty, a padded place of the batch)."""
    n, longest = case["seqs"], case["longest"]
    if not case.get("ragged"):
        return [longest] * n
    rng = random.Random(n * 1000003 + longest)
    lens = [longest] + [rng.randint(1, longest) for _ in range(n - 1)]
    if n >= 8:
        lens[n // 2] = 0
    return lens


# --------------------------------------------------------------------------
# rotary frequencies: base 10000 and the usual scalings of long contexts
# --------------------------------------------------------------------------
_SCALING = {
    "none": dict(),
    "linear": dict(factor=4.0),
    "yarn": dict(factor=8.0, original_length=8192, beta_fast=32.0, beta_slow=1.0),
    "llama3": dict(factor=8.0, original_length=8192, low_freq_factor=1.0, high_freq_factor=4.0),
}
_BASE = 500000.0


def _frequencies(rotary, scaling):
    """Radians per token of each pair, in 64 bits, and the factor on cosine and sine."""
    a = _SCALING[scaling]
    i = torch.arange(rotary // 2, dtype=torch.float64, device="cuda")
    f = _BASE ** (-2.0 * i / rotary)
    if scaling == "linear":
        return f / a["factor"], 1.0
    if scaling == "yarn":
        # between the pairs that make beta_fast and beta_slow turns over the original length: from f to f / factor
        lo, hi = (rotary * math.log(a["original_length"] / (turns * 2 * math.pi)) / (2 * math.log(_BASE))
                  for turns in (a["beta_fast"], a["beta_slow"]))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rotary - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / a["factor"] * ramp + f * (1 - ramp), 0.1 * math.log(a["factor"]) + 1.0
    if scaling == "llama3":
        # below low_freq_factor turns over the original length: f / factor; above high_freq_factor: f
        turns = a["original_length"] * f / (2 * math.pi)
        keep = ((turns - a["low_freq_factor"]) / (a["high_freq_factor"] - a["low_freq_factor"])).clamp(0, 1)
        return (1 - keep) * f / a["factor"] + keep * f, 1.0
    return f, 1.0


def _rotate(x, positions, freqs, m, rotary, interleaved, backward=False):
    """The rotation of x [T, H, D] in 32 bits (angles in 64), as 32 bits."""
    angle = positions.double()[:, None] * freqs
    c = (angle.cos() * m).float()[:, None, :]
    s = (angle.sin() * m).float()[:, None, :]
    if backward:
        s = -s
    y = x.float()
    if interleaved:
        a, b = y[..., 0:rotary:2], y[..., 1:rotary:2]
        r = torch.stack((a * c - b * s, a * s + b * c), dim=-1).flatten(-2)
    else:
        a, b = y[..., :rotary // 2], y[..., rotary // 2:rotary]
        r = torch.cat((a * c - b * s, a * s + b * c), dim=-1)
    return torch.cat((r, y[..., rotary:]), dim=-1)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) + 1)
    return g


def _keys(g, shape, dtype, big=8.0):
    """Unit normal with a few large channels, as keys have (big = 1: values, queries)."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16 if dtype == torch.float16 else torch.float32)
    if big != 1.0:
        x[..., torch.randperm(shape[-1], generator=g, device="cuda")[:max(1, shape[-1] // 50)]] *= big
    return x.to(dtype)


def _pages(case, g, lens, spare=3):
    """A block table that gives each sequence its pages, spread over the pool; a row's places past its length
    are -1.  (table int32 [seqs, most], pages in the pool)"""
    page, need = case["page"], [-(-n // case["page"]) for n in lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device="cuda", dtype=torch.int32)
    table = torch.full((len(lens), max(1, -(-case["longest"] // page))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total


def _encode(x, group_s):
    """Eq. 1 and Eq. 2 on fp16 x [rows, D]: packed codes, FLAGs, scales.  In 32 bits, as both are defined."""
    rows, D = x.shape
    xg = x.float().view(rows, D // 64, 64)
    # a true division, also where a compiler would multiply by the reciprocal of a constant
    s = (xg.abs().amax(-1, keepdim=True) / torch.full((1,), 127.0, device=x.device)).half()
    r = torch.where(s > 0, 1.0 / s.float(), torch.zeros_like(s, dtype=torch.float32))
    q = (xg * r).round().clamp(-127, 127).view(rows, D // group_s, group_s).to(torch.int16)
    m = q.abs().amax(-1, keepdim=True)
    flag = (m >= 8).to(torch.int16) + (m >= 16) + (m >= 32) + (m >= 64)
    c = (torch.sign(q) * (q.abs() >> flag)).view(rows, D // 2, 2) & 15
    return (c[..., 0] | (c[..., 1] << 4)).to(torch.uint8), flag.view(rows, -1).to(torch.uint8), s.view(rows, -1)


def _decode(codes, flags, scales):
    """32-bit values [rows, D] of encoded rows (a product of 3 and 11 bits: exact)."""
    rows, half = codes.shape
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(rows, 2 * half).to(torch.int32)
    c = torch.where(c >= 8, c - 16, c).view(rows, flags.shape[1], -1)
    v = (c << flags.to(torch.int32)[..., None]).float()
    return (v.view(rows, scales.shape[1], -1) * scales.float()[..., None]).view(rows, 2 * half)


def _pool(case, g, total, big):
    """One side (keys or values) of a filled pool: a 16-bit tensor [pages, page, heads, D], or encoded rows
    (page, head, slot) as (codes, flags, scales)."""
    H, page, D = case.get("kv_heads", case.get("heads")), case["page"], case["dim"]
    if case["store"] != "lzs":
        dtype = _DTYPES[case["store"]]
        if case["heads_first"]:
            return _keys(g, (total, H, page, D), dtype, big).transpose(1, 2)
        return _keys(g, (total, page, H, D), dtype, big)
    rows = total * H * page
    out = [torch.empty((rows, D // 2), dtype=torch.uint8, device="cuda"),
           torch.empty((rows, D // case["group_s"]), dtype=torch.uint8, device="cuda"),
           torch.empty((rows, D // 64), dtype=torch.float16, device="cuda")]
    step = 2 ** 25 // D
    for i in range(0, rows, step):
        for t, e in zip(out, _encode(_keys(g, (min(step, rows - i), D), torch.float16, big), case["group_s"])):
            t[i:i + step] = e
    return tuple(out)


def _inputs(case, seed):
    """What the call gets, as plain tensors."""
    g = _gen(seed)
    if case["kind"] == "rope":
        T, H, D = case["tokens"], case["heads"], case["dim"]
        extra = 2 if case["fused"] else 0  # two more heads (a key's and a value's) behind the queries'
        x = _keys(g, (T, H + extra, D), _DTYPES[case["dtype"]], 1.0)[:, :H]
        start = max(0, case["far"] - T)
        pos = torch.randint(0, start + 1, (1,), generator=g, device="cuda") + torch.arange(T, device="cuda")
        return dict(x=x, positions=pos)
    lens = _lens(case)
    H, page, D = case.get("kv_heads", case.get("heads")), case["page"], case["dim"]
    table, total = _pages(case, g, lens)
    d = dict(table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             k=_pool(case, g, total, 8.0), v=_pool(case, g, total, 1.0))
    if case["kind"] == "append":
        n, T = case["new"], case["seqs"] * case["new"]
        dtype = torch.float16 if case["store"] == "lzs" else _DTYPES[case["store"]]
        at = torch.arange(case["longest"] - n, case["longest"], device="cuda").repeat(case["seqs"], 1)
        d["positions"] = at.reshape(-1)
        d["slots"] = (table.long().gather(1, at // page) * page + at % page).reshape(-1)
        d["new_k"], d["new_v"] = _keys(g, (T, H, D), dtype, 8.0), _keys(g, (T, H, D), dtype, 1.0)
    elif case["kind"] == "attend":
        out = torch.float16 if case["store"] == "lzs" else _DTYPES[case["store"]]
        d["q"] = _keys(g, (case["seqs"], case["q_heads"], D), out, 1.0)
        if case["weights"]:
            d["weights"] = torch.rand((case["seqs"], H, table.shape[1] * page), generator=g, device="cuda")
    else:
        # sums of softmax weights: a wide spread, the first token large, and many that were never looked at
        n = table.shape[1] * page
        w = torch.exp(1.5 * torch.randn((case["seqs"], H, n), generator=g, device="cuda"))
        w *= torch.rand((case["seqs"], H, n), generator=g, device="cuda") < 0.95
        w[..., 0] = 50.0
        d["weights"] = w
        d["new_table"], extra = _pages(dict(case, longest=case["budget"]), g, [min(x, case["budget"]) for x in lens])
        d["new_table"] = torch.where(d["new_table"] >= 0, d["new_table"] + total, d["new_table"])
        # the pool goes on behind the sequences' pages with those that the kept rows go to
        for side in ("k", "v"):
            old = d[side]
            if case["heads_first"]:
                new = torch.zeros((total + extra, H, page, D), dtype=old.dtype, device="cuda").transpose(1, 2)
            else:
                new = torch.zeros((total + extra, page, H, D), dtype=old.dtype, device="cuda")
            new[:total] = old
            d[side] = new
    return d


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["kind"] == "rope":
        s["freqs"], s["m"] = _frequencies(case["rotary"], case["scaling"])
    elif case.get("rope"):
        s["freqs"], s["m"] = _frequencies(case["dim"], "llama3")
    if own and case["kind"] != "rope":  # the handle of a cache that a program keeps
        import paper_2509_26436_gb300 as Q
        k, v = s["k"], s["v"]
        if case["store"] == "lzs":
            p = Q.Params(group_s=case["group_s"])
            k, v = (Q.Encoded(*side, None, None, side[0].shape[0], case["dim"], p) for side in (k, v))
        s["cache"] = Q.PagedCache(k, v, case["page"], case.get("kv_heads", case.get("heads")))
    return s


# --------------------------------------------------------------------------
# a pass
# --------------------------------------------------------------------------
def _rows(case, side, table, t, heads):
    """The rows of the tokens t [seqs, n] (places in their sequences) as 32-bit values [seqs, heads, n, D]; those
    without a page are some other token's."""
    page = case["page"]
    p, j = table.long().gather(1, t // page).clamp(min=0), t % page
    if case["store"] != "lzs":
        return side[p, j].transpose(1, 2).float()
    at = (p[:, None] * heads + torch.arange(heads, device="cuda")[:, None]) * page + j[:, None]
    return _decode(side[0][at].flatten(0, 2), side[1][at].flatten(0, 2), side[2][at].flatten(0, 2)).view(
        *at.shape, case["dim"])


def _run_rope(s):
    case = s["case"]
    y = _rotate(s["x"], s["positions"], s["freqs"], s["m"], case["rotary"], case["interleaved"], case["backward"])
    return y.to(s["x"].dtype)


def _run_append(s):
    case, H, page = s["case"], s["case"]["heads"], s["case"]["page"]
    k, v, slots = s["new_k"], s["new_v"], s["slots"]
    if case["rope"]:
        k = _rotate(k, s["positions"], s["freqs"], s["m"], case["dim"], False).to(k.dtype)
    if case["store"] != "lzs":
        s["k"][slots // page, slots % page] = k
        s["v"][slots // page, slots % page] = v
        return dict(k=s["k"], v=s["v"])
    at = ((slots[:, None] // page * H + torch.arange(H, device="cuda")) * page + slots[:, None] % page).reshape(-1)
    for side, x in ((s["k"], k), (s["v"], v)):
        for t, e in zip(side, _encode(x.reshape(-1, case["dim"]), case["group_s"])):
            t[at] = e
    return dict(k=_decode(*s["k"]).half(), v=_decode(*s["v"]).half())


def _run_attend(s):
    case, w = s["case"], s.get("weights")
    B, Hq, H, D = case["seqs"], case["q_heads"], case["kv_heads"], case["dim"]
    longest = case["longest"]
    n = min(longest, case["window"]) if case["window"] else longest
    lens = s["lens"].long()[:, None]
    t = (lens - n).clamp(min=0) + torch.arange(n, device="cuda")
    seen = (t < lens)[:, None, None]
    t = t.clamp(max=longest - 1)
    q = s["q"].float().view(B, H, Hq // H, D)
    score = torch.matmul(q, _rows(case, s["k"], s["table"], t, H).transpose(2, 3)) * D ** -0.5
    score = score.masked_fill(~seen, -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    p = e / e.sum(-1, keepdim=True).clamp(min=1e-30)  # an empty sequence has no weights
    o = torch.matmul(p, _rows(case, s["v"], s["table"], t, H)).view(B, Hq, D).to(_DTYPES[case["out"]])
    if w is None:
        return o
    return dict(o=o, weights=w.scatter_add(2, t[:, None].expand(-1, H, -1), p.sum(2)))


def _run_evict(s):
    case, weights, page = s["case"], s["weights"], s["case"]["page"]
    B, H, N = weights.shape
    budget = case["budget"]
    t = torch.arange(N, device="cuda")
    lens = s["lens"].long()[:, None, None]
    score = weights.masked_fill((t < case["sinks"]) | (t >= lens - case["recent"]), math.inf)
    score = torch.where(lens > budget, score, weights).masked_fill(t >= lens, -math.inf)
    # a stable sort leaves equal weights in the order of their tokens
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.full((B, H, budget), N, dtype=torch.int64, device="cuda")
    j = torch.arange(budget, device="cuda")
    m = lens.clamp(max=budget)
    kept[..., :best.shape[-1]] = best
    kept = kept.masked_fill(j >= m, N).sort(-1).values
    b, h, j = (j < m).expand(-1, H, -1).nonzero(as_tuple=True)
    old = kept[b, h, j]
    src, dst = s["table"].long()[b, old // page], s["new_table"].long()[b, j // page]
    s["k"][dst, j % page, h] = s["k"][src, old % page, h]
    s["v"][dst, j % page, h] = s["v"][src, old % page, h]
    left = weights.masked_fill(t < lens, 0)
    left[b, h, j] = weights[b, h, old]
    return dict(kept=kept.masked_fill(kept == N, -1).int(), lens=s["lens"].clamp(max=budget), k=s["k"], v=s["v"],
                weights=left)


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"rope": _run_rope, "append": _run_append, "attend": _run_attend, "evict": _run_evict}[case["kind"]](s)
    import paper_2509_26436_gb300 as Q
    if case["kind"] == "rope":
        return Q.rope(s["x"], s["positions"], s["freqs"], interleaved=case["interleaved"], scale=s["m"],
                      backward=case["backward"])
    cache = s["cache"]
    if case["kind"] == "append":
        if case["rope"]:
            Q.paged_append(cache, s["new_k"], s["new_v"], s["slots"], positions=s["positions"], freqs=s["freqs"],
                           rope_scale=s["m"])
        else:
            Q.paged_append(cache, s["new_k"], s["new_v"], s["slots"])
        if case["store"] == "lzs":
            return dict(k=Q.dequantize(cache.k), v=Q.dequantize(cache.v))
        return dict(k=cache.k, v=cache.v)
    if case["kind"] == "attend":
        scale, out = case["dim"] ** -0.5, _DTYPES[case["out"]]
        if not case["weights"]:
            return Q.attention_paged(s["q"], cache, s["table"], s["lens"], scale, window=case["window"],
                                     out_dtype=out)
        w = s["weights"].clone()  # the sums so far stay as they were for the next pass
        o = Q.attention_paged(s["q"], cache, s["table"], s["lens"], scale, window=case["window"], out_dtype=out,
                              weights=w)
        return dict(o=o, weights=w)
    kept, lens = Q.evict_select(s["weights"], s["lens"], case["budget"], recent=case["recent"], sinks=case["sinks"])
    w = s["weights"].clone()
    Q.cache_compact(cache, s["table"], s["lens"], kept, lens, new_table=s["new_table"], weights=w)
    return dict(kept=kept, lens=lens, k=cache.k, v=cache.v, weights=w)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def _stored(case):
    """Bytes of one token's key and value of one head in the cache."""
    D = case["dim"]
    return 2 * (D / 2 + D / case["group_s"] + D / 32) if case["store"] == "lzs" else 4 * D


def work(case):
    D = case["dim"]
    if case["kind"] == "rope":
        size = {"float16": 2, "bfloat16": 2, "float32": 4}[case["dtype"]]
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * D * size + 8 * case["tokens"], "flops": 3 * n * case["rotary"]}
    if case["kind"] == "append":
        T = case["seqs"] * case["new"]
        b = T * case["heads"] * (4 * D + _stored(case)) + T * (16 if case["rope"] else 8)
        f = T * case["heads"] * D * 5
        if case["store"] == "lzs":  # the whole pool read back
            rows = (case["seqs"] * -(-case["longest"] // case["page"]) + 3) * case["page"] * case["heads"]
            b, f = b + rows * (_stored(case) + 4 * D), f + 2 * rows * D
        return {"bytes": b, "flops": f}
    lens = _lens(case)
    H = case["kv_heads"]
    if case["kind"] == "attend":
        out = {"float16": 2, "bfloat16": 2, "float32": 4}[case["out"]]
        seen = sum(min(n, case["window"]) if case["window"] else n for n in lens)
        b = seen * H * _stored(case) + case["seqs"] * (case["q_heads"] * D * (2 + out) + 4)
        b += 4 * sum(-(-n // case["page"]) for n in lens)
        if case["weights"]:
            b += 8 * seen * H
        return {"bytes": b, "flops": 4 * seen * case["q_heads"] * D}
    rows = sum(min(n, case["budget"]) for n in lens) * H
    b = 4 * sum(lens) * H + 4 * rows + 2 * rows * _stored(case) + 4 * sum(lens) * H
    return {"bytes": b, "flops": sum(lens) * H}


# --------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------
def _turned(x, positions, rotary, interleaved, scaling, backward):
    """Each pair as a complex number, times m e^(i angle) (backward: its conjugate)."""
    freqs, m = _frequencies(rotary, scaling)
    z = torch.polar(torch.full((positions.numel(), rotary // 2), m, dtype=torch.float64, device="cuda"),
                    positions.double()[:, None] * freqs)[:, None]
    x = x.double()
    part = x[..., :rotary]
    if interleaved:
        pairs = torch.complex(part[..., 0::2], part[..., 1::2])
    else:
        pairs = torch.complex(*part.chunk(2, dim=-1))
    pairs = pairs * (z.conj() if backward else z)
    y = x.clone()
    if interleaved:
        y[..., 0:rotary:2], y[..., 1:rotary:2] = pairs.real, pairs.imag
    else:
        y[..., :rotary // 2], y[..., rotary // 2:rotary] = pairs.real, pairs.imag
    return y


def _held(case, side, heads):
    """What the pool stands for, in 64 bits: [pages, page, heads, D]."""
    if case["store"] != "lzs":
        return side.double()
    page, D = case["page"], case["dim"]
    byte = side[0].to(torch.int16)
    c = torch.stack((byte & 15, byte >> 4), dim=-1).double().flatten(1)
    c = c - 16 * (c > 7)
    c = c * (1 << side[1].to(torch.int32)).repeat_interleave(case["group_s"], dim=1)
    c = c * side[2].double().repeat_interleave(64, dim=1)
    return c.view(-1, heads, page, D).transpose(1, 2)


def _exact_append(case, d):
    H, D, page = case["heads"], case["dim"], case["page"]
    new = [d["new_k"].double(), d["new_v"].double()]
    if case["rope"]:
        new[0] = _turned(d["new_k"], d["positions"], D, False, "llama3", False)
    out = []
    for side, x in zip((d["k"], d["v"]), new):
        y = _held(case, side, H).clone()
        if case["store"] == "lzs":
            x = x.half().double()  # what the encoder gets is 16 bits wide
            g = x.view(-1, D // 64, 64)
            s = (g.abs().amax(-1, keepdim=True) / 127).half().double()
            r = (1 / s.clamp(min=2.0 ** -24)).float().double()  # x / s is defined as x r, both rounded to 32 bits
            q = torch.where(s > 0, (g * r).float().double().round(), g * 0).clamp(-127, 127)
            q = q.view(-1, D // case["group_s"], case["group_s"])
            bits = torch.frexp(q.abs().amax(-1, keepdim=True)).exponent
            unit = torch.ldexp(torch.ones_like(q[..., :1]), (bits - 3).clamp(min=0))
            x = ((q / unit).trunc() * unit).view_as(g) * s
            x = x.view(-1, H, D)
        y[d["slots"] // page, d["slots"] % page] = x
        out.append(y)
    if case["store"] == "lzs":  # as the cache's rows: (page, head, slot)
        out = [y.transpose(1, 2).reshape(-1, D) for y in out]
    return dict(k=out[0], v=out[1])


def _exact_attend(case, d):
    B, Hq, H, D, page = case["seqs"], case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    o = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda")
    w = d["weights"].double() if case["weights"] else None
    for b, n in enumerate(_lens(case)):
        if n == 0:
            continue
        pages = d["table"][b, :-(-n // page)].long()
        sides = []
        for side in (d["k"], d["v"]):
            if case["store"] == "lzs":
                at = (pages[:, None] * (H * page) + torch.arange(H * page, device="cuda")).reshape(-1)
                held = _held(case, tuple(t[at] for t in side), H)
            else:
                held = side[pages].double()
            sides.append(held.reshape(-1, H, D)[:n])
        k, v = sides
        seen = torch.arange(n, device="cuda") >= (n - case["window"] if case["window"] else 0)
        for h in range(H):
            for r in range(h * (Hq // H), (h + 1) * (Hq // H)):
                score = (k[:, h] @ d["q"][b, r].double()) / math.sqrt(D)
                p = torch.softmax(score.masked_fill(~seen, -math.inf), 0)
                o[b, r] = p @ v[:, h]
                if w is not None:
                    w[b, h, :n] += p
    return o if w is None else dict(o=o, weights=w)


def _exact_evict(case, d):
    page, budget, H = case["page"], case["budget"], case["kv_heads"]
    k, v, w = d["k"].clone(), d["v"].clone(), d["weights"].double()
    held = d["weights"].cpu().numpy()
    for b, n in enumerate(_lens(case)):
        m = min(n, budget)
        for h in range(H):
            keep = np.arange(n)
            if n > budget:
                mid = np.arange(case["sinks"], n - case["recent"])
                order = np.lexsort((mid, -held[b, h, mid].astype(np.float64)))
                best = mid[order[:budget - case["sinks"] - case["recent"]]]
                keep = np.sort(np.concatenate((np.arange(case["sinks"]), best, np.arange(n - case["recent"], n))))
            keep = torch.from_numpy(keep).to(d["table"].device)
            j = torch.arange(m, device="cuda")
            src, dst = d["table"][b].long()[keep // page], d["new_table"][b].long()[j // page]
            k[dst, j % page, h] = k[src, keep % page, h]
            v[dst, j % page, h] = v[src, keep % page, h]
            w[b, h, :m] = d["weights"][b, h, keep].double()
            w[b, h, m:n] = 0
    return dict(kept=None, lens=None, k=k.double(), v=v.double(), weights=w)


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "rope":
        return _turned(d["x"], d["positions"], case["rotary"], case["interleaved"], case["scaling"], case["backward"])
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["kind"]](case, d)
