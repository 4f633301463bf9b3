"""Operators for several new tokens per sequence, as they are timed: the norm of each head's queries and keys with the
position rotation in the same pass (and its gradient), rotary positions with several axes, and attention of prompts and
of trees of drafted tokens over a paged cache.

A case is one pass of an operator.  With `own` false a pass is the operator's definition in elementary torch
operations, in 32 bits (angles and long sums in 64); with `own` true it is the package's call.  exact() restates the
definitions in 64 bits, apart from both.
"""
import math
import random

import torch

own = False

_DTYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}
_EPS = 1e-6


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _named(name, c):
    return dict(c, name=name) if name else c


def _norm(name, tokens, q_heads, k_heads, dim, rotary, dtype, axes=1, interleaved=False, weights="same", fused=True,
          backward=False):
    return _named(name, dict(kind="norm", tokens=tokens, q_heads=q_heads, k_heads=k_heads, dim=dim, rotary=rotary,
                             dtype=dtype, axes=axes, interleaved=interleaved, weights=weights, fused=fused,
                             backward=backward))


def _axes(name, tokens, heads, dim, rotary, dtype, axes, interleaved=False, dealt=False, backward=False):
    return _named(name, dict(kind="axes", tokens=tokens, heads=heads, dim=dim, rotary=rotary, dtype=dtype, axes=axes,
                             interleaved=interleaved, dealt=dealt, backward=backward))


def _attend(name, seqs, q_heads, kv_heads, dim, context, new, ragged, page, store, group_s=16, tree=False, window=0,
            cap=0.0, slopes=False, prefix=0, heads_first=False):
    return _named(name, dict(kind="attend", seqs=seqs, q_heads=q_heads, kv_heads=kv_heads, dim=dim, context=context,
                             new=new, ragged=ragged, page=page, store=store, group_s=group_s, tree=tree,
                             window=window, cap=cap, slopes=slopes, prefix=prefix, heads_first=heads_first))


def listed():
    return [
        # queries and keys of one decode step, 16 sequences: latency alone
        _norm("norm_step", 16, 32, 8, 128, 128, "bfloat16"),
        # an image of 64 x 64 patches behind 512 words of text, 24 heads, three axes, as the projection left them
        _norm("norm_image", 4608, 24, 24, 128, 128, "float16", axes=3, interleaved=True),
        # the gradient of a training step, with respect to queries, keys and both norms' weights
        _norm("norm_grad", 8192, 32, 8, 128, 128, "bfloat16", weights="float32", backward=True),
        # odd heads of which a part is turned, 32-bit gradients, an odd token count
        _norm("norm_grad_partial", 1999, 20, 4, 96, 64, "float32", fused=False, backward=True),
        # frames x rows x columns of a video's patches, pairs dealt to the axes in turn
        _axes("axes_video", 13 * 30 * 45, 16, 128, 128, "bfloat16", 3, dealt=True),
        # a small picture's rows and columns, the gradient, heads of 72
        _axes("axes_picture_grad", 729, 16, 72, 72, "float16", 2, interleaved=True, backward=True),
        # eight drafted tokens of one conversation, every query head with its own keys: latency
        _attend("tree_one_777", 1, 40, 40, 128, 777, 8, False, 16, "float16", tree=True),
        # a batch verifying trees of 16 drafted tokens over contexts of all lengths
        _attend("tree_batch", 16, 32, 8, 128, 8192, 16, True, 16, "bfloat16", tree=True),
        # large trees over long contexts in 4-bit pages, eight query heads to a key head
        _attend("tree_long_lzs", 4, 64, 8, 128, 65536, 61, True, 64, "lzs", tree=True),
        # a long prompt, causal
        _attend("prompt_long", 1, 32, 8, 128, 0, 8192, False, 64, "bfloat16"),
        # chunks of prompts behind what is cached already, 4-bit pages, scores capped
        _attend("prompt_chunk_lzs", 4, 32, 8, 128, 8192, 509, True, 32, "lzs", group_s=8, cap=50.0),
        # wide heads, a window, a prefix that all see, distances in the scores
        _attend("prompt_window_256", 3, 16, 4, 256, 2048, 1777, True, 16, "float16", window=1024, slopes=True,
                prefix=130, heads_first=True),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    what = rng.choice(["norm"] * 3 + ["axes"] + ["attend"] * 6)
    if what != "attend":
        dim = rng.choice([64, 72, 80, 96, 128, 128, 192, 256])
        rotary = rng.choice([dim, dim, dim, dim // 2])
        dtype = rng.choice(["float16", "bfloat16", "bfloat16", "float32"])
        axes = rng.choice([1, 1, 2, 3])
        most = 8192 * 40 * 128 // (2 if dtype == "float32" else 1)
        if what == "norm":
            kh = _log(rng, 1, 24)
            qh = kh * rng.choice([1, 2, 4, 5, 8])
            tokens = _log(rng, 1, max(1, min(32768, most // (dim * (qh + kh)))))
            return _norm(None, tokens, qh, kh, dim, rotary, dtype, axes, rng.random() < 0.4,
                         rng.choice(["same", "float32", "none"]), rng.random() < 0.7, rng.random() < 0.5)
        heads = _log(rng, 1, 48)
        tokens = _log(rng, 1, max(1, min(65536, most // (dim * heads))))
        return _axes(None, tokens, heads, dim, rotary, dtype, rng.choice([2, 3]), rng.random() < 0.4,
                     rng.random() < 0.5, rng.random() < 0.4)
    dim = rng.choice([64, 128, 128, 128, 192, 256])
    store = rng.choice(["float16", "bfloat16", "lzs"])
    gs = rng.choice([8, 16, 16, 32, 64])
    kv = _log(rng, 1, 16)
    qh = kv * rng.choice([1, 2, 3, 4, 5, 8])
    page = rng.choice([8, 16, 32, 64, 128])
    tree = rng.random() < 0.45
    seqs = _log(rng, 1, 32 if tree else 12)
    new = _log(rng, 1, 64 if tree else 4096)
    # what the longest prompt costs, and half a gigabyte of 16-bit pages
    ops = 2 ** 37 // (qh * dim * seqs)
    most = min(65536, 2 ** 28 // (2 * kv * dim * seqs), ops // new)
    while most < new and new > 1:
        new //= 2
        most = min(65536, 2 ** 28 // (2 * kv * dim * seqs), ops // new)
    context = _log(rng, 1, max(1, most - new)) - 1
    window = rng.choice([0, 0, 0, rng.randrange(64, context + new + 128)])
    prefix = rng.choice([0, 0, 0, rng.randrange(1, context + new + 1)])
    return _attend(None, seqs, qh, kv, dim, context, new, rng.random() < 0.7, page, store, gs, tree, window,
                   rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), rng.random() < 0.25, prefix, rng.random() < 0.3)


def _counts(case):
    """(lengths, new tokens) of the sequences: of the case alone.  Ragged ones spread over the whole range (one is the
    longest, and of three or more one has no new token at all)."""
    n = case["seqs"]
    if not case["ragged"]:
        return [case["context"] + case["new"]] * n, [case["new"]] * n
    rng = random.Random(n * 1000003 + case["context"] * 101 + case["new"])
    new = [case["new"]] + [rng.randint(1, case["new"]) for _ in range(n - 1)]
    lens = [case["context"] + new[0]] + [rng.randint(0, case["context"]) + new[i] for i in range(1, n)]
    if n >= 3:
        lens[n // 2], new[n // 2] = lens[n // 2] - new[n // 2], 0
    return lens, new


def _trees(case):
    """The drafted tokens each drafted token sees, as bits (itself and its ancestors), for every sequence."""
    rng = random.Random(case["seqs"] * 7919 + case["new"])
    out = []
    for n in _counts(case)[1]:
        masks = []
        for j in range(n):
            parent = rng.randrange(-1, j) if j % 4 == 0 else (rng.randrange(j) if j else -1)
            masks.append((masks[parent] if parent >= 0 else 0) | (1 << j))
        out.append(masks)
    return out


def _prefixes(case):
    rng = random.Random(case["seqs"] * 31 + case["prefix"])
    return [rng.randint(0, case["prefix"]) if i else case["prefix"] for i in range(case["seqs"])]


# --------------------------------------------------------------------------
# rotary frequencies and positions of several axes
# --------------------------------------------------------------------------
_BASE = 10000.0


def _pairs(case):
    """(radians per position of each pair in 64 bits, each pair's axis).  Runs of pairs per axis, each with a spectrum
    of its own, or one spectrum whose pairs are dealt to the axes in turn."""
    n, axes = case["rotary"] // 2, case["axes"]
    if axes == 1:
        return [_BASE ** (-i / n) for i in range(n)], [0] * n
    if case.get("dealt"):
        return [_BASE ** (-i / n) for i in range(n)], [i % axes for i in range(n)]
    first = n // 8 if axes == 3 else n // 2  # time, or text: fewer pairs than rows and columns
    rest = n - first
    sizes = [first, rest] if axes == 2 else [first, rest // 2, rest - rest // 2]
    freqs, axis = [], []
    for a, m in enumerate(sizes):
        freqs += [_BASE ** (-i / m) for i in range(m)]
        axis += [a] * m
    return freqs, axis


def _positions(case, seed):
    """int64 [axes, tokens]: places in a grid (or a line), from a place of the seed on."""
    T = case["tokens"]
    t = torch.arange(T, device="cuda")
    at = random.Random(seed).randrange(4096)
    if case["axes"] == 1:
        return (t + at)[None].contiguous()
    side = max(1, int(math.sqrt(T)))
    if case["axes"] == 2:
        return torch.stack((t // side, t % side))
    side = max(1, int(T ** (1 / 3)))
    return torch.stack((t // (side * side) + at % 64, t // side % side, t % side))


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) + 1)
    return g


def _normal(g, shape, dtype, big=1.0):
    """Unit normal; with a few large channels, as keys have, where `big` is not 1."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16 if dtype == torch.float16 else torch.float32)
    if big != 1.0:
        x[..., torch.randperm(shape[-1], generator=g, device="cuda")[:max(1, shape[-1] // 50)]] *= big
    return x.to(dtype)


def _encode(x, group_s):
    """8-bit codes per group of 64, cut to 4 bits per subgroup: packed codes, FLAGs, scales of fp16 x [rows, D]."""
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


def _pool(case, g, total, big):
    """One side of a filled pool: a 16-bit tensor [pages, page, heads, D], or encoded rows (page, head, slot) as
    (codes, FLAGs, scales)."""
    H, page, D = case["kv_heads"], case["page"], case["dim"]
    if case["store"] != "lzs":
        dtype = _DTYPES[case["store"]]
        if case["heads_first"]:
            return _normal(g, (total, H, page, D), dtype, big).transpose(1, 2)
        return _normal(g, (total, page, H, D), dtype, big)
    rows = total * H * page
    out = [torch.empty((rows, D // 2), dtype=torch.uint8, device="cuda"),
           torch.empty((rows, D // case["group_s"]), dtype=torch.uint8, device="cuda"),
           torch.empty((rows, D // 64), dtype=torch.float16, device="cuda")]
    step = 2 ** 25 // D
    for i in range(0, rows, step):
        for t, e in zip(out, _encode(_normal(g, (min(step, rows - i), D), torch.float16, big), case["group_s"])):
            t[i:i + step] = e
    return tuple(out)


def _inputs(case, seed):
    """What the call gets, as plain tensors."""
    g = _gen(seed)
    D = case["dim"]
    if case["kind"] == "axes":
        dtype = _DTYPES[case["dtype"]]
        return dict(x=_normal(g, (case["tokens"], case["heads"], D), dtype), positions=_positions(case, seed))
    if case["kind"] == "norm":
        T, Hq, Hk = case["tokens"], case["q_heads"], case["k_heads"]
        dtype = _DTYPES[case["dtype"]]
        d = dict(positions=_positions(case, seed), wq=None, wk=None)
        if case["fused"]:  # queries, keys and values side by side, as one projection writes them
            x = _normal(g, (T, Hq + 2 * Hk, D), dtype, 4.0)
            d["q"], d["k"] = x[:, :Hq], x[:, Hq:Hq + Hk]
        else:
            d["q"], d["k"] = _normal(g, (T, Hq, D), dtype, 4.0), _normal(g, (T, Hk, D), dtype, 4.0)
        if case["weights"] != "none":
            w = torch.float32 if case["weights"] == "float32" else dtype
            d["wq"], d["wk"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(w) for _ in range(2))
        if case["backward"]:
            d["dq"], d["dk"] = _normal(g, (T, Hq, D), dtype), _normal(g, (T, Hk, D), dtype)
        return d
    lens, new = _counts(case)
    page, need = case["page"], [-(-n // case["page"]) for n in lens]
    total = sum(need) + 3
    order = torch.randperm(total, generator=g, device="cuda", dtype=torch.int32)
    table = torch.full((len(lens), max(1, -(-max(lens) // page))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    dtype = torch.float16 if case["store"] == "lzs" else _DTYPES[case["store"]]
    d = dict(table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
             q=_normal(g, (starts[-1], case["q_heads"], D), dtype),
             k=_pool(case, g, total, 8.0), v=_pool(case, g, total, 1.0))
    if case["tree"]:
        # bit 63 is the sign of 64-bit integers
        masks = [m - (1 << 64) if m >> 63 else m for seq in _trees(case) for m in seq]
        d["tree"] = torch.tensor(masks, dtype=torch.int64, device="cuda")
    if case["prefix"]:
        d["prefix"] = torch.tensor(_prefixes(case), dtype=torch.int32, device="cuda")
    if case["slopes"]:  # 2^(-8 h / heads), the usual geometric series
        h = torch.arange(1, case["q_heads"] + 1, device="cuda", dtype=torch.float64)
        d["slopes"] = (2.0 ** (-8.0 * h / case["q_heads"])).float()
    return d


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["kind"] != "attend":
        freqs, axis = _pairs(case)
        s["freqs"] = torch.tensor(freqs, dtype=torch.float64, device="cuda")
        s["axis"] = torch.tensor(axis, dtype=torch.int32, device="cuda")
    elif own:  # the handle of a cache that a program keeps
        import paper_2509_26436_gb300 as Q
        k, v = s["k"], s["v"]
        if case["store"] == "lzs":
            p = Q.Params(group_s=case["group_s"])
            k, v = (Q.Encoded(*side, None, None, side[0].shape[0], case["dim"], p) for side in (k, v))
        s["cache"] = Q.PagedCache(k, v, case["page"], case["kv_heads"])
    return s


# --------------------------------------------------------------------------
# a pass
# --------------------------------------------------------------------------
def _cos_sin(s):
    """[tokens, 1, pairs], angles in 64 bits."""
    angle = s["positions"][s["axis"].long()].t().double() * s["freqs"]
    return angle.cos().float()[:, None], angle.sin().float()[:, None]


def _rotate(x, c, s, rotary, interleaved):
    """32-bit x [T, H, D] with its first `rotary` elements turned."""
    if interleaved:
        a, b = x[..., 0:rotary:2], x[..., 1:rotary:2]
        r = torch.stack((a * c - b * s, a * s + b * c), dim=-1).flatten(-2)
    else:
        a, b = x[..., :rotary // 2], x[..., rotary // 2:rotary]
        r = torch.cat((a * c - b * s, a * s + b * c), dim=-1)
    return torch.cat((r, x[..., rotary:]), dim=-1)


def _run_axes(s):
    case = s["case"]
    c, sn = _cos_sin(s)
    y = _rotate(s["x"].float(), c, -sn if case["backward"] else sn, case["rotary"], case["interleaved"])
    return y.to(s["x"].dtype)


def _run_norm(s):
    case = s["case"]
    c, sn = _cos_sin(s)
    out = {}
    for side in ("q", "k"):
        x, w = s[side].float(), s["w" + side]
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
        weight = 1.0 if w is None else w.float()
        if not case["backward"]:
            out[side] = _rotate(x * r * weight, c, sn, case["rotary"], case["interleaved"]).to(s[side].dtype)
            continue
        g = _rotate(s["d" + side].float(), c, -sn, case["rotary"], case["interleaved"])  # of the normed, weighted head
        n = x * r
        gw = g * weight
        out["d" + side] = (r * (gw - n * (gw * n).mean(-1, keepdim=True))).to(s[side].dtype)
        if w is not None:
            out["dw" + side] = (g * n).double().sum((0, 1)).to(w.dtype)
    return out


def _decode(codes, flags, scales):
    """What encoded rows stand for, rounded to fp16 as a key or value is, in 32 bits [rows, D]."""
    rows, half = codes.shape
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(rows, 2 * half).to(torch.int32)
    c = torch.where(c >= 8, c - 16, c).view(rows, flags.shape[1], -1)
    v = (c << flags.to(torch.int32)[..., None]).float()
    return (v.view(rows, scales.shape[1], -1) * scales.float()[..., None]).view(rows, 2 * half).half().float()


def _rows(case, side, pages, n):
    """The first n tokens of the given pages as 32-bit values [heads, n, D]."""
    page, H, D = case["page"], case["kv_heads"], case["dim"]
    if case["store"] != "lzs":
        return side[pages].flatten(0, 1)[:n].transpose(0, 1).float()
    t = torch.arange(n, device="cuda")
    at = ((pages[t // page] * H)[None] + torch.arange(H, device="cuda")[:, None]) * page + t % page
    return _decode(*(x[at.reshape(-1)] for x in side)).view(H, n, D)


def _run_attend(s):
    case = s["case"]
    Hq, H, D, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    G = Hq // H
    o = torch.empty_like(s["q"])
    at = 0
    for b, (n, m) in enumerate(zip(*_counts(case))):
        if m == 0:
            continue
        pages = s["table"][b, :-(-n // page)].long()
        k, v = _rows(case, s["k"], pages, n), _rows(case, s["v"], pages, n)
        q = s["q"][at:at + m].float().view(m, H, G, D).permute(1, 2, 0, 3)  # [H, G, m, D]
        t = torch.arange(n, device="cuda")
        j = torch.arange(m, device="cuda")
        base = n - m
        if case["tree"]:
            bits = (s["tree"][at:at + m, None] >> j) & 1  # [token, token it sees]
            depth = (bits.sum(-1) - 1).clamp(min=0)
            pos, place = base + depth, torch.cat((t[:base], base + depth))
            seen = torch.cat((torch.ones((m, base), dtype=torch.bool, device="cuda"), bits.bool()), dim=1)
        else:
            pos, place = base + j, t
            seen = t <= pos[:, None]
        if case["window"]:
            seen = seen & (place > pos[:, None] - case["window"])
        if case["prefix"]:
            seen = seen | (t < s["prefix"][b])
        step = max(1, 2 ** 28 // (G * m * n))  # key heads at a time
        for h in range(0, H, step):
            score = torch.matmul(q[h:h + step], k[h:h + step, None].transpose(2, 3)) * D ** -0.5
            if case["cap"]:
                score = case["cap"] * torch.tanh(score / case["cap"])
            if case["slopes"]:
                slope = s["slopes"][h * G:(h + step) * G].view(-1, G, 1, 1)
                score = score - slope * (place - pos[:, None]).abs().float()
            score = score.masked_fill(~seen, -math.inf)
            e = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
            p = e / e.sum(-1, keepdim=True).clamp(min=1e-30)  # a token that sees nothing has no weights
            r = torch.matmul(p, v[h:h + step, None])
            o[at:at + m].view(m, H, G, D)[:, h:h + step] = r.permute(2, 0, 1, 3).to(o.dtype)
        at += m
    return o


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"axes": _run_axes, "norm": _run_norm, "attend": _run_attend}[case["kind"]](s)
    import paper_2509_26436_gb300 as Q
    if case["kind"] == "axes":
        return Q.rope_axes(s["x"], s["positions"], s["freqs"], s["axis"], interleaved=case["interleaved"],
                           backward=case["backward"])
    if case["kind"] == "norm":
        how = dict(eps=_EPS, interleaved=case["interleaved"])
        if case["axes"] == 1:
            positions = s["positions"][0]
        else:
            positions, how["pair_axis"] = s["positions"], s["axis"]
        if not case["backward"]:
            q, k = Q.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], positions, s["freqs"], **how)
            return dict(q=q, k=k)
        dq, dk, dwq, dwk = Q.qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], positions,
                                                   s["freqs"], **how)
        out = dict(dq=dq, dk=dk)
        if s["wq"] is not None:
            out.update(dwq=dwq, dwk=dwk)
        return out
    return Q.attention_paged_tokens(s["q"], s["cache"], s["table"], s["lens"], s["starts"], case["dim"] ** -0.5,
                                    tree=s.get("tree"), prefix_lens=s.get("prefix"), window=case["window"],
                                    cap=case["cap"], slopes=s.get("slopes"), max_new=case["new"])


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def _seen(case):
    """For each sequence with new tokens: (pairs of new and seen tokens, cached tokens that any of them sees)."""
    out = []
    trees, prefixes = (_trees(case) if case["tree"] else None), _prefixes(case)
    for b, (n, m) in enumerate(zip(*_counts(case))):
        if m == 0:
            continue
        base, w, pre = n - m, case["window"], min(prefixes[b], n)
        pairs, low = 0, n
        for j in range(m):
            if case["tree"]:
                depth = bin(trees[b][j]).count("1") - 1
                first = max(0, base + depth - w + 1) if w else 0
                own_tokens = sum(1 for i in range(m) if (trees[b][j] >> i) & 1 or base + i < pre)
                pairs += max(0, base - max(first, pre)) + min(pre, base) + own_tokens
            else:
                first, end = (max(0, base + j - w + 1) if w else 0), base + j + 1
                pairs += max(0, end - max(first, pre)) + pre
            low = min(low, first)
        out.append((pairs, n - max(0, low - pre)))
    return out


def work(case):
    D = case["dim"]
    size = {"float16": 2, "bfloat16": 2, "float32": 4}.get(case.get("dtype"))
    if case["kind"] == "axes":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * D * size + 8 * case["axes"] * case["tokens"], "flops": 3 * n * case["rotary"]}
    if case["kind"] == "norm":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"])
        if case["backward"]:
            return {"bytes": 3 * n * D * size + 8 * case["axes"] * case["tokens"], "flops": n * (12 * D + 3 * case["rotary"])}
        return {"bytes": 2 * n * D * size + 8 * case["axes"] * case["tokens"], "flops": n * (5 * D + 3 * case["rotary"])}
    stored = 2 * (D / 2 + D / case["group_s"] + D / 32) if case["store"] == "lzs" else 4 * D
    pairs = sum(p for p, _ in _seen(case))
    read = sum(r for _, r in _seen(case))
    b = read * case["kv_heads"] * stored + 4 * sum(_counts(case)[1]) * case["q_heads"] * D
    return {"bytes": b, "flops": 4 * pairs * case["q_heads"] * D}


# --------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------
def _turned(x, case, positions, backward):
    """Each pair of 64-bit x [T, H, D] as a complex number, times e^(i angle) (backward: its conjugate)."""
    n = case["rotary"] // 2
    freqs, axis = _pairs(case)
    angle = torch.stack([positions[a].double() * f for f, a in zip(freqs, axis)], dim=1)
    z = torch.polar(torch.ones_like(angle), -angle if backward else angle)[:, None]
    i = torch.arange(n, device=x.device)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + n)
    pairs = torch.complex(x[..., first], x[..., second]) * z
    y = x.clone()
    y[..., first], y[..., second] = pairs.real, pairs.imag
    return y


def _exact_norm(case, d):
    out = {}
    for side in ("q", "k"):
        x = d[side].double()
        w = torch.ones(case["dim"], dtype=torch.float64, device="cuda") if d["w" + side] is None else d["w" + side].double()
        length = (x.square().sum(-1, keepdim=True) / case["dim"] + _EPS).sqrt()
        if not case["backward"]:
            out[side] = _turned(x / length * w, case, d["positions"], False)
            continue
        g = _turned(d["d" + side].double(), case, d["positions"], True)
        # d(x_i / length) = dx_i / length - x_i (x . dx) / (D length^3)
        along = (g * w * x).sum(-1, keepdim=True) / (case["dim"] * length ** 3)
        out["d" + side] = g * w / length - x * along
        if d["w" + side] is not None:
            out["dw" + side] = (g * x / length).sum((0, 1))
    return out


def _exact_attend(case, d):
    Hq, H, D, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    o = torch.zeros((d["q"].shape[0], Hq, D), dtype=torch.float64, device="cuda")
    trees, prefixes = _trees(case), _prefixes(case)
    at = 0
    for b, (n, m) in enumerate(zip(*_counts(case))):
        if m == 0:
            continue
        base = n - m
        pos = [base + (bin(trees[b][j]).count("1") - 1 if case["tree"] else j) for j in range(m)]
        place = torch.tensor(list(range(base)) + pos, device="cuda")
        own_seen = torch.zeros((m, m), dtype=torch.bool)
        for j in range(m):
            if case["tree"]:
                own_seen[j] = torch.tensor([(trees[b][j] >> i) & 1 == 1 for i in range(m)])
            else:
                own_seen[j, :j + 1] = True
        allowed = torch.ones((m, n), dtype=torch.bool, device="cuda")
        allowed[:, base:] = own_seen.cuda()
        distance = (torch.tensor(pos, device="cuda")[:, None] - place).double()
        if case["window"]:
            allowed &= distance < case["window"]
        allowed[:, :prefixes[b] if case["prefix"] else 0] = True
        pages = d["table"][b, :-(-n // page)].long()
        held = []
        for side in (d["k"], d["v"]):
            if case["store"] != "lzs":
                held.append(side[pages].double().reshape(-1, H, D)[:n])
                continue
            rows = (pages[:, None] * (H * page) + torch.arange(H * page, device="cuda")).reshape(-1)
            byte = side[0][rows].to(torch.int16)
            c = torch.stack((byte & 15, byte >> 4), dim=-1).double().flatten(1)
            c = (c - 16 * (c > 7)) * torch.pow(2.0, side[1][rows].double()).repeat_interleave(case["group_s"], dim=1)
            c = (c * side[2][rows].double().repeat_interleave(64, dim=1)).half().double()
            held.append(c.view(-1, H, page, D).transpose(1, 2).reshape(-1, H, D)[:n])
        for r in range(Hq):
            score = d["q"][at:at + m, r].double() @ held[0][:, r * H // Hq].t() / math.sqrt(D)
            if case["cap"]:
                score = torch.tanh(score / case["cap"]) * case["cap"]
            if case["slopes"]:
                score -= d["slopes"][r].double() * distance.abs()
            score.masked_fill_(~allowed, -math.inf)
            p = torch.nan_to_num(torch.softmax(score, dim=-1), nan=0.0)
            o[at:at + m, r] = p @ held[1][:, r * H // Hq]
        at += m
    return o


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "axes":
        return _turned(d["x"].double(), case, d["positions"], case["backward"])
    return _exact_norm(case, d) if case["kind"] == "norm" else _exact_attend(case, d)
