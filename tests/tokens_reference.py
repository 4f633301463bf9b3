"""The operators for several new tokens per sequence from their definitions, in 64
bits on the CPU, with bounds on what binary32 arithmetic may be off by."""
import torch

import paged_reference as R

U = 2.0 ** -24  # half a step of binary32


def rope_axes(x, positions, freqs, axis, interleaved=False, scale=1.0, backward=False):
    """Pair by pair: a rotation of one pair by its axis's positions."""
    y = x.double().clone()
    n = len(freqs)
    for i in range(n):
        i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        pair = R.rope(x[..., [i1, i2]], positions[axis[i]], freqs[i:i + 1], False, scale, backward)
        y[..., i1], y[..., i2] = pair[..., 0], pair[..., 1]
    return y


def _turn(x, positions, freqs, axis, interleaved, scale, backward):
    if freqs is None:
        return x.double().clone()
    if axis is None:
        return R.rope(x, positions, freqs, interleaved, scale, backward)
    return rope_axes(x, positions, freqs, axis, interleaved, scale, backward)


def turn_bound(ax, relative, positions, freqs, axis, interleaved, scale):
    """What a binary32 rotation of values of size `ax`, each off by `relative` of
    itself already, may be off by: paged_reference.rope_bound without the last
    rounding, per pair; elements that are not turned keep their own error."""
    b = ax * relative
    if freqs is None:
        return b
    n = len(freqs)
    i = torch.arange(n)
    i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    pair = ax[..., i1] + ax[..., i2]
    at = positions[None].expand(n, -1) if axis is None else positions[torch.tensor(axis)]  # [pair, token]
    turns = freqs.double() / (2 * torch.pi)
    err = 2 * torch.pi * at.t().double().abs() * (turns * 1.5 * 2.0 ** -53 + 2.0 ** -64)
    t = abs(scale) * pair * (relative + err[:, None] + 5 * U)
    b[..., i1], b[..., i2] = t, t
    return b


def rounded(bound, y, dtype):
    info = torch.finfo(dtype)
    return bound + info.eps / 2 * (y.abs() + bound) + info.smallest_normal * info.eps / 2


def norm(x, w, eps, positions, freqs, axis, interleaved, scale):
    """(y, its binary32 bound).  The sum of D squares: D rounded products and
    additions, so D + 1 half steps of it, half as much of its root's
    reciprocal; division by D and eps: 3; rsqrtf: 2 steps, that is 4; r w and
    its product with x: 2."""
    x = x.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double()
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    nw = x * r * w
    relative = ((x.shape[-1] + 4) / 2 + 4 + 2) * U
    return _turn(nw, positions, freqs, axis, interleaved, scale, False), \
        turn_bound(nw.abs(), relative, positions, freqs, axis, interleaved, scale)


def norm_grad(x, w, dy, eps, positions, freqs, axis, interleaved, scale):
    """(dx, dw, bound of dx, bound of dw), as norm()."""
    D = x.shape[-1]
    x, dy = x.double(), dy.double()
    w = torch.ones(D, dtype=torch.float64) if w is None else w.double()
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    g = _turn(dy, positions, freqs, axis, interleaved, scale, True)
    n = x * r
    along = r * (g * w * n).mean(-1, keepdim=True)  # dx = r (g w - x along)
    dx = r * (g * w - x * along)
    dw = (g * n).sum((0, 1))
    e_g = turn_bound(dy.abs(), 0.0, positions, freqs, axis, interleaved, scale)
    e_r = ((D + 4) / 2 + 4) * U
    size = (g * w * x).abs().sum(-1, keepdim=True)
    e_along = r ** 2 / D * (((w * x).abs() * e_g).sum(-1, keepdim=True) + size * ((D + 4) * U + 2 * e_r))
    e_dx = r * (w.abs() * e_g + x.abs() * e_along) + r * ((g * w).abs() + (x * along).abs()) * (e_r + 4 * U)
    # the sum over rows: in whatever order, at most as many half steps as there are rows
    rows = x.shape[0] * x.shape[1]
    e_dw = (n.abs() * e_g + (g * n).abs() * (e_r + (3 + rows) * U)).sum((0, 1))
    return dx, dw, e_dx, e_dw


# --- attention ----------------------------------------------------------------
def places(n, m, tree=None):
    """(positions of the m new tokens, places of the n cached ones)."""
    base = n - m
    if tree is None:
        pos = [base + j for j in range(m)]
        return pos, list(range(n))
    pos = [base + max(0, bin(t & ((1 << m) - 1)).count("1") - 1) for t in tree]
    return pos, list(range(base)) + pos


def seen(n, m, tree=None, window=0, prefix=0):
    """bool [m, n], from the definition, token by token."""
    base = n - m
    pos, place = places(n, m, tree)
    out = torch.zeros((m, n), dtype=torch.bool)
    t = torch.arange(n)
    at = torch.tensor(place, dtype=torch.int64)
    for j in range(m):
        s = t <= pos[j] if tree is None else (t < base)
        if tree is not None and m:
            s[base:] = torch.tensor([(tree[j] >> i) & 1 == 1 for i in range(m)])
        if window:
            s = s & (at > pos[j] - window)
        out[j] = s | (t < prefix)
    return out


def attention(q, k, v, scale, mask, dtype, pos=None, place=None, cap=0.0, slopes=None):
    """(o, bound) of one sequence: q [m, Hq, D], k and v [n, H, D], mask [m, n].

    A score is off by its products' sum, D + 1 half steps of binary32 of the sum
    of their sizes, doubled since the tensor cores cut where binary32 rounds;
    8 half steps of itself for its factors (a cap: 25 of the capped score, and a
    capped score moves by no more than the score), 4 of the distance's product
    (of up to 128 more) and the result.  A weight is off by that, by 2^-22 (ex2) and by half a step
    of the pages' type (relative to the largest: fp16 holds weights from 2^-22
    of the largest down to 2^-33 of it); sums of n weights, or of n products,
    by n + 2 half steps, doubled for the tensor cores, and the rescaling and the
    join by 16 more."""
    m, Hq, D = q.shape
    n, H, _ = k.shape
    G = Hq // H
    o, bound = torch.zeros((m, Hq, D), dtype=torch.float64), torch.zeros((m, Hq, D), dtype=torch.float64)
    if n == 0:
        return o, bound
    info = torch.finfo(dtype)
    for h in range(Hq):
        kk, vv = k[:, h // G].double(), v[:, h // G].double()
        qq = q[:, h].double()
        # what is not seen may be anything
        some = mask.any(0)
        kk, vv = (torch.where(some[:, None], x, torch.zeros_like(x)) for x in (kk, vv))
        s = qq @ kk.t() * scale
        size = qq.abs() @ kk.abs().t() * abs(scale)
        err = size * 2 * (D + 1) * U + s.abs() * 8 * U
        if cap:
            s = cap * torch.tanh(s / cap)
            err = err + s.abs() * 25 * U
        if slopes is not None:
            far = (pos[:, None] - place[None]).abs().double() * float(slopes[h])
            s = s - far
            # the distance from a tile of 128 keys' first one is rounded by itself
            err = err + (far.abs() + 128 * abs(float(slopes[h]))) * 4 * U + s.abs() * 4 * U
        s = s.masked_fill(~mask, -torch.inf)
        top = s.amax(-1, keepdim=True).clamp(min=-1e300)
        e = torch.exp(s - top)
        total = e.sum(-1, keepdim=True)
        p = torch.where(total > 0, e / total.clamp(min=1e-300), torch.zeros_like(e))
        err = torch.where(mask, err, torch.zeros_like(err))
        # the running maximum that all are relative to is off as well: by the largest error
        rel = err + err.amax(-1, keepdim=True) * 2 ** -20 + (s - top).abs().nan_to_num(0, 0, 0) * 4 * U + 2.0 ** -22
        rel = rel * 1.01 + info.eps / 2
        small = 2.0 ** -33 if dtype == torch.float16 else 0.0
        a = p @ vv.abs()
        sums = (2 * (n + 2) + 16) * U
        o[:, h] = p @ vv
        low = torch.where(mask, torch.full_like(p, small), torch.zeros_like(p)) @ vv.abs()
        # numerator, and the denominator's part: the weights' own errors without the rounding, as l is not rounded
        den = (p * (rel - info.eps / 2)).sum(-1, keepdim=True) + sums
        bound[:, h] = (p * rel) @ vv.abs() + a * (sums + den) * 1.01 + low
    return o, bound
