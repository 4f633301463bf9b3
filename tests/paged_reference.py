"""The paged cache's operators from their definitions, in 64 bits on the CPU,
for the tests: nothing here is shared with the package."""
import math
from fractions import Fraction

import numpy as np
import torch

# pi to 60 digits
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def angles(positions, freqs):
    """positions x freqs radians, reduced to [0, 2 pi) without rounding: float64."""
    out = np.empty((len(positions), len(freqs)))
    for j, f in enumerate(freqs):
        turn = Fraction(float(f)) / (2 * PI)
        for i, p in enumerate(positions):
            x = turn * int(p)
            out[i, j] = float((x - math.floor(x)) * 2 * PI)
    return torch.from_numpy(out)


def rope(x, positions, freqs, interleaved=False, scale=1.0, backward=False):
    a = angles(positions.tolist(), freqs.tolist())[:, None]
    c, s = a.cos() * scale, a.sin() * scale
    if backward:
        s = -s
    y = x.double().clone()
    n = len(freqs)
    i = torch.arange(n)
    i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    x1, x2 = y[..., i1].clone(), y[..., i2].clone()
    y[..., i1] = c * x1 - s * x2
    y[..., i2] = s * x1 + c * x2
    return y


def rope_bound(x, positions, freqs, interleaved, scale, dtype, y):
    """How far a binary32 rotation rounded to `dtype` may be from y.

    Angle: the frequency in turns carries 1.5 * 2^-53 of its size (the 64-bit
    product and the constant) and what lies below 2^-64, times the position;
    the last conversion 2^-24 of at most an eighth of a turn.  Sine and cosine:
    one ulp (2^-24) each, the factor half an ulp; products and sum half an ulp
    each: in all at most 5 * 2^-24 of |x1| + |x2|.  Then the rounding to the
    type: half a step, or half the smallest subnormal."""
    n = len(freqs)
    i = torch.arange(n)
    i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    ax = x.double().abs()
    pair = ax[..., i1] + ax[..., i2]
    turns = freqs.double() / (2 * math.pi)
    err = 2 * math.pi * positions.double().abs()[:, None] * (turns * 1.5 * 2.0 ** -53 + 2.0 ** -64)
    b = abs(scale) * pair * (err[:, None] + 5 * 2.0 ** -24)
    bound = torch.zeros_like(ax)
    bound[..., i1], bound[..., i2] = b, b
    info = torch.finfo(dtype)
    return bound + info.eps / 2 * (y.abs() + bound) + info.smallest_normal * info.eps / 2


def decode(codes, flags, scales):
    """Encoded rows as 64-bit values [rows, D]."""
    byte = codes.to(torch.int64)
    c = torch.stack((byte & 15, byte >> 4), -1).flatten(1)
    c = torch.where(c > 7, c - 16, c)
    rows, D = c.shape
    v = (c.view(rows, flags.shape[1], -1) * (1 << flags.to(torch.int64))[..., None]).view(rows, scales.shape[1], -1)
    return (v.double() * scales.double()[..., None]).view(rows, D)


def held(cache):
    """(k, v) of a cache as 64-bit [pages, page_size, heads, dim] on the CPU."""
    out = []
    for side in (cache.k, cache.v):
        if hasattr(side, "codes"):
            d = decode(side.codes.cpu(), side.flags.cpu(), side.scales.cpu())
            out.append(d.view(cache.num_pages, cache.heads, cache.page_size, cache.dim).transpose(1, 2))
        else:
            out.append(side.cpu().double())
    return out


def attention(q, k, v, table, lens, scale, window=0):
    """o [B, Hq, D], weights' additions [B, H, most], and for the bounds the
    largest sum |q_d k_d| scale a head sees [B, Hq], sum p |v| [B, Hq, D]."""
    q = q.double()
    B, Hq, D = q.shape
    page, H = k.shape[1], k.shape[2]
    most = table.shape[1] * page
    o, mag = torch.zeros(B, Hq, D, dtype=torch.float64), torch.zeros(B, Hq, dtype=torch.float64)
    pv = torch.zeros(B, Hq, D, dtype=torch.float64)
    add = torch.zeros(B, H, most, dtype=torch.float64)
    for b, n in enumerate(lens.tolist()):
        first = max(0, n - window) if window else 0
        if n == 0:
            continue
        t = torch.arange(first, n)
        pages = table[b].long()[t // page]
        kb, vb = k[pages, t % page], v[pages, t % page]
        for r in range(Hq):
            h = r // (Hq // H)
            s = kb[:, h] @ q[b, r] * scale
            p = torch.softmax(s, 0)
            o[b, r] = p @ vb[:, h]
            pv[b, r] = p @ vb[:, h].abs()
            mag[b, r] = (kb[:, h].abs() @ q[b, r].abs()).max() * abs(scale)
            add[b, h, first:n] += p
    return o, add, mag, pv


def attention_bounds(mag, pv, o, add, tokens, D, group, out_dtype, pair_bits, most_v):
    """Bounds on o and on the weights' additions (relative).

    A score is a sum of D exact products accumulated in binary32 (each step
    may truncate: 2^-23 of the magnitudes' sum), times group scale and softmax
    scale (2^-23 more each), minus the maximum (2^-23 of both): eps_p = (D + 8)
    2^-23 mag nats, and 2^-22 for the exponential.  The weights enter the value
    product in two parts of `pair_bits` together.  Sums over the tokens: at
    most tokens / 16 + 64 steps a chain, 2^-23 each, in numerator and
    denominator.  Weights below binary32's smallest normal number, 2^-126, may
    become 0, and so may what a weight times a group scale leaves below it,
    which multiplies a code's value of at most 112: an absolute 2^-126 (|v| +
    112) per token, divided by a denominator of at least 1 (the largest weight
    counts as 1).  Then the output's rounding."""
    eps_p = (D + 8) * 2.0 ** -23 * mag + 2.0 ** -22
    chain = (tokens / 16 + 64) * 2.0 ** -23
    rel = 2 * eps_p + 2.0 ** -pair_bits + 2 * chain
    info = torch.finfo(out_dtype)
    bound = rel[..., None] * pv + tokens * 2.0 ** -126 * (most_v + 112)
    bound = bound + info.eps / 2 * (o.abs() + bound) + info.smallest_normal * info.eps / 2
    B, Hq = mag.shape
    w_rel = (2 * eps_p + chain + group * 2.0 ** -23).view(B, -1, group).amax(-1)
    return bound, w_rel


def evict(weights, lens, budget, recent, sinks):
    """kept [B, H, budget] (numpy int32) and the new lengths."""
    w = weights.cpu().numpy()
    B, H, _ = w.shape
    kept = np.full((B, H, budget), -1, np.int32)
    for b, n in enumerate(lens.tolist()):
        for h in range(H):
            if n <= budget:
                kept[b, h, :n] = np.arange(n)
                continue
            middle = range(sinks, n - recent)
            key = sorted(middle, key=lambda t: (-w[b, h, t] if w[b, h, t] == w[b, h, t] else math.inf, t))
            # NaN comes last of all, behind -inf
            real = [t for t in key if w[b, h, t] == w[b, h, t]]
            nan = [t for t in key if w[b, h, t] != w[b, h, t]]
            best = (real + nan)[:budget - sinks - recent]
            kept[b, h] = sorted(list(range(sinks)) + best + list(range(n - recent, n)))
    return torch.from_numpy(kept), torch.clamp(lens.cpu(), max=budget)
