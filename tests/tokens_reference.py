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
