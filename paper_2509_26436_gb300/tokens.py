"""Several new tokens per sequence: the norm of each head's queries and keys with
the rotary positions in the same pass (and its gradient), rotary positions of
several axes, and attention of prompts and of trees of drafted tokens over a
paged cache.

As paged.py, whose cache and frequencies these go with, this only marshals torch
CUDA tensors into the C ABI; every call is asynchronous on the current stream
(or `stream`), and nothing is recorded for autograd: a tensor whose gradient
would be lost is refused.

    freqs, scale = rope_frequencies(128, base=500000.0)
    q, k = qk_norm_rope(q, k, wq, wk, positions, freqs, scale=scale)
    paged_append(cache, k, v, slots)
    o = attention_paged_tokens(q, cache, block_table, seq_lens, starts, 128 ** -0.5)
    dq, dk, dwq, dwk = qk_norm_rope_backward(gq, gk, q, k, wq, wk, positions, freqs, scale=scale)
"""
from __future__ import annotations

import ctypes as C

import paper_2509_26436_gb300 as _Q

from . import _native as N
from . import paged as P

_byref = C.byref
_TREE_MOST = 64  # drafted tokens of a sequence: bits of a mask


def _no_gradient(name, instead, *tensors):
    for t in tensors:
        if t is not None and t.requires_grad:
            raise ValueError(f"{name} records no gradient: use torch.no_grad(), or {instead}")


_FUNCTION = "an autograd function whose backward calls "


def _axes_struct(positions, freqs, pair_axis, tokens, scale, interleaved, backward, device) -> N.QuartzRopeAxes:
    """positions [tokens] (one axis), or [axes, tokens] with pair_axis."""
    pairs = freqs.shape[0]
    f = P._vector("freqs", freqs, P.f64, device)
    if pair_axis is None:
        at, stride, axes, pa = P._vector("positions", positions, P.i64, device), 0, 1, None
    else:
        stride = P._rows("positions", positions, 2, P.i64, device)[0]
        at, axes, pa = positions.data_ptr(), positions.shape[0], P._vector("pair_axis", pair_axis, P.i32, device)
        if pair_axis.shape[0] != pairs:
            raise ValueError("pair_axis must have one entry per frequency")
    if positions.shape[-1] != tokens:
        raise ValueError("positions must have one entry per token")
    return N.QuartzRopeAxes(at, stride, f, pa, axes, 2 * pairs, interleaved, backward, scale)


def rope_axes(x, positions, freqs, pair_axis, interleaved: bool = False, scale: float = 1.0, backward: bool = False,
              out=None, stream=None):
    """rope() by positions of several axes (time, row and column of an image's
    or a video's patches): x [tokens, heads, dim <= 256], positions int64 [axes,
    tokens], and pair i turned by positions[pair_axis[i], t] * freqs[i], with
    pair_axis int32 [len(freqs)] on the device.  Types, strides, `out` and
    gradients as in rope()."""
    if P.torch is None:
        P._bind()
    if P.torch.is_grad_enabled():
        _no_gradient("rope_axes", _FUNCTION + "rope_axes(..., backward=True)", x, out, freqs)
    dtype = x.dtype
    kind = P._KIND.get(dtype)
    if kind is None or not x.is_cuda:
        raise ValueError("x must be a 3-D float16, bfloat16 or float32 CUDA tensor")
    device = P._device()
    xs = P._rows("x", x, 3, dtype, device)
    T, H, D = x.shape
    if pair_axis is None:
        raise ValueError("pair_axis must name the axis of each frequency (one axis: rope())")
    r = _axes_struct(positions, freqs, pair_axis, T, scale, interleaved, backward, device)
    if out is None:
        out = P._empty((T, H, D), dtype, x.device, stream)
        s0, s1 = H * D, D
    else:
        s0, s1, _ = P._rows("out", out, 3, dtype, device)
        if out.shape != x.shape:
            raise ValueError("out must have the shape of x")
    rc = P.lib.quartz_rope_axes(x.data_ptr(), xs[0], xs[1], out.data_ptr(), s0, s1, kind, T, H, D, _byref(r),
                                _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_rope_axes")
    return out


def _norm_types(q, wq, wk):
    """(type of q and k, of the weights, and both as the ABI's)."""
    dtype = q.dtype
    w_dtype = wq.dtype if wq is not None else wk.dtype if wk is not None else dtype
    kind, w_kind = P._KIND.get(dtype), P._KIND.get(w_dtype)
    if kind is None or not q.is_cuda or q.dim() != 3:
        raise ValueError("q must be a 3-D float16, bfloat16 or float32 CUDA tensor")
    if w_kind is None or (wk is not None and wk.dtype is not w_dtype):
        raise ValueError("wq and wk must be float16, bfloat16 or float32, of one type")
    return dtype, w_dtype, kind, w_kind


def _norm_side(name, x, w, T, D, dtype, w_dtype, device):
    """(strides, heads and address of x, address of w) after the checks of one
    side.  (P._rows and P._vector in line: a call's host time is mostly these.)"""
    st = x.stride()
    if x.dtype is not dtype or len(st) != 3 or x.get_device() != device or (st[2] != 1 and x.shape[-1] > 1):
        P._refuse(name, x, 3, dtype)
    tokens, heads, dim = x.shape
    if tokens != T or dim != D:
        raise ValueError("q and k must have the same tokens and dim")
    if w is None:
        return st[0], st[1], heads, x.data_ptr(), None
    if w.dtype is not w_dtype or w.dim() != 1 or w.get_device() != device or not w.is_contiguous():
        P._refuse("w" + name, w, 1, w_dtype)
    if w.shape[0] != D:
        raise ValueError(f"w{name} must have one entry per element of a head")
    return st[0], st[1], heads, x.data_ptr(), w.data_ptr()


def _rope_of(positions, freqs, pair_axis, T, scale, interleaved, device):
    if positions is None and freqs is None:
        return None
    if positions is None or freqs is None:
        raise ValueError("positions and freqs go together")
    return _byref(_axes_struct(positions, freqs, pair_axis, T, scale, interleaved, False, device))


def _norm_out(x, y, T, H, D, dtype, device, stream):
    """The result (given, or new) with its strides."""
    if y is None:
        return P._empty((T, H, D), dtype, x.device, stream), H * D, D
    y0, y1, _ = P._rows("out", y, 3, dtype, device)
    if y.shape != x.shape:
        raise ValueError("out must have the shapes of q and k")
    return y, y0, y1


def qk_norm_rope(q, k, wq, wk, positions=None, freqs=None, eps: float = 1e-6, pair_axis=None, interleaved: bool = False,
                 scale: float = 1.0, out=None, stream=None):
    """(yq, yk): the norm of each head of q [tokens, q_heads, dim] and k [tokens,
    k_heads, dim] (or None), x (mean x^2 + eps)^-1/2 w, then rope()'s rotation
    of its first 2 len(freqs) elements by positions int64 [tokens], or with
    pair_axis rope_axes()'s by positions [axes, tokens]; no positions and freqs:
    no rotation.  float16, bfloat16 or float32, any strides with a contiguous
    last dimension (views of a fused projection), dim <= 256; wq and wk [dim] in
    one of these types, or None: ones.  In binary32, rounded once.  `out` (yq,
    yk) may be (q, k).  Nothing is recorded for autograd (rope())."""
    if P.torch is None:
        P._bind()
    if P.torch.is_grad_enabled():
        _no_gradient("qk_norm_rope", _FUNCTION + "qk_norm_rope_backward", q, k, wq, wk, freqs, *(out or ()))
    dtype, w_dtype, kind, w_kind = _norm_types(q, wq, wk)
    device = P._device()
    T, Hq, D = q.shape
    x0, x1, _, x_ptr, w_ptr = _norm_side("q", q, wq, T, D, dtype, w_dtype, device)
    yq, yk = (None, None) if out is None else out
    yq, y0, y1 = _norm_out(q, yq, T, Hq, D, dtype, device, stream)
    side_q = N.QuartzNormSide(x_ptr, x0, x1, None, 0, 0, yq.data_ptr(), y0, y1, w_ptr, None, Hq)
    if k is None:
        side_k, yk = N.QuartzNormSide(), None
    else:
        x0, x1, Hk, x_ptr, w_ptr = _norm_side("k", k, wk, T, D, dtype, w_dtype, device)
        yk, y0, y1 = _norm_out(k, yk, T, Hk, D, dtype, device, stream)
        side_k = N.QuartzNormSide(x_ptr, x0, x1, None, 0, 0, yk.data_ptr(), y0, y1, w_ptr, None, Hk)
    r = _rope_of(positions, freqs, pair_axis, T, scale, interleaved, device)
    rc = P.lib.quartz_qk_norm_rope(_byref(side_q), _byref(side_k), kind, w_kind, T, D, eps, r, _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_qk_norm_rope")
    return yq, yk


def qk_norm_rope_backward(dyq, dyk, q, k, wq, wk, positions=None, freqs=None, eps: float = 1e-6, pair_axis=None,
                          interleaved: bool = False, scale: float = 1.0, workspace=None, stream=None):
    """(dq, dk, dwq, dwk): the gradients of qk_norm_rope's q, k, wq and wk (None
    for what is None) from those of its results (of their types and shapes, any
    strides with a contiguous last dimension) and the same arguments.  The weights' gradients are summed in
    binary32 in the same order on every call.  Nothing is recorded for autograd,
    for a second derivative neither (rope()).  A workspace of the caller's
    (qk_norm_rope_workspace_size bytes) is only good for one call at a time, and
    for one captured graph."""
    if P.torch is None:
        P._bind()
    if P.torch.is_grad_enabled():
        _no_gradient("qk_norm_rope_backward", "detach what it gets", dyq, dyk, q, k, wq, wk, freqs)
    dtype, w_dtype, kind, w_kind = _norm_types(q, wq, wk)
    device = P._device()
    T, _, D = q.shape
    sides, grads = [], []
    for name, x, dy, w in (("q", q, dyq, wq), ("k", k, dyk, wk)):
        if x is None:
            if dy is not None or w is not None:
                raise ValueError(f"{name} is None, and has neither a gradient nor weights")
            sides.append(N.QuartzNormSide())
            grads += (None, None)
            continue
        x0, x1, H, x_ptr, w_ptr = _norm_side(name, x, w, T, D, dtype, w_dtype, device)
        if dy is None or dy.shape != x.shape:
            raise ValueError(f"dy{name} must have the shape of {name}")
        ds = P._rows("dy" + name, dy, 3, dtype, device)
        dx, y0, y1 = _norm_out(x, None, T, H, D, dtype, device, stream)
        dw = None if w is None else P._empty((D,), w_dtype, x.device, stream)
        sides.append(N.QuartzNormSide(x_ptr, x0, x1, dy.data_ptr(), ds[0], ds[1], dx.data_ptr(), y0, y1, w_ptr,
                                      None if w is None else dw.data_ptr(), H))
        grads += (dx, dw)
    ptr, size = None, 0
    if wq is not None or wk is not None:
        if workspace is None:
            size = P.lib.quartz_qk_norm_rope_workspace_size(D)
            workspace = P._empty((size,), P.torch.uint8, q.device, stream)
        else:
            if workspace.get_device() != device or not workspace.is_contiguous():
                raise ValueError("workspace must be a contiguous CUDA tensor on the current device")
            size = workspace.numel() * workspace.element_size()
        ptr = workspace.data_ptr()
    r = _rope_of(positions, freqs, pair_axis, T, scale, interleaved, device)
    rc = P.lib.quartz_qk_norm_rope_backward(_byref(sides[0]), _byref(sides[1]), kind, w_kind, T, D, eps, r, ptr, size,
                                            _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_qk_norm_rope_backward")
    return grads[0], grads[2], grads[1], grads[3]


def qk_norm_rope_workspace_size(dim: int) -> int:
    return N.load().quartz_qk_norm_rope_workspace_size(dim)


# --- attention ----------------------------------------------------------------

def attention_paged_tokens(q, cache: P.PagedCache, block_table, seq_lens, starts, scale: float, tree=None,
                           prefix_lens=None, window: int = 0, cap: float = 0.0, slopes=None, max_len: int | None = None,
                           max_new: int | None = None, out_dtype=None, out=None, workspace=None, stream=None):
    """o [tokens, q_heads, dim]: attention of the new tokens of several sequences,
    side by side in q [tokens, q_heads, dim] (the cache's type; float16 for
    encoded pages), over the paged cache, in which they are the last of their
    sequence already (paged_append).  Rows starts[b] to starts[b + 1] are
    sequence b's (starts int32 [seqs + 1]; a sequence may have none); rows
    before the first and behind the last are left as they are in `out`.
    seq_lens int32 [seqs]: cached tokens, the new ones among them.

    Each sees the tokens up to its own position; with `window` > 0 only those
    less than `window` before it; and the first prefix_lens[b] tokens whatever
    their position (int32 [seqs]).  `tree` int64 [tokens]: bit i of a row says
    that it sees its sequence's drafted token i (itself too, by its own bit),
    besides the tokens before them all; the position is then that of the first
    drafted token plus the number of other drafted tokens that it sees.  Scores:
    scale q . k; cap > 0: cap tanh(score / cap); slopes float32 [q_heads]: less
    slopes[h] times the distance of the positions.  A token that sees nothing
    gives zeros.

    max_len: at most this many cached tokens (default: what the table holds),
    max_new: at most this many new ones per sequence (default: all of q; 64 in
    a tree, which holds no more); known bounds plan better.  Softmax weights
    multiply the values as two parts of the cache's type where a key head has at
    most 128 rows (max_new times its query heads) or the result is float32;
    else rounded to that type.  A workspace of the caller's is only good for one
    call at a time, and for one captured graph.  Nothing is recorded for autograd
    (rope())."""
    if P.torch.is_grad_enabled():
        _no_gradient("attention_paged_tokens", "detach what it gets", q, slopes, out, *cache._pools)
    device = cache._check_device()
    qs = P._rows("q", q, 3, cache.dtype, device)
    ts = P._rows("block_table", block_table, 2, P.i32, device)
    lens, at = P._vector("seq_lens", seq_lens, P.i32, device), P._vector("starts", starts, P.i32, device)
    T, Hq, D = q.shape
    B, width = block_table.shape
    if D != cache.dim or Hq % cache.heads or seq_lens.shape[0] != B or starts.shape[0] != B + 1:
        raise ValueError("q must be [tokens, a multiple of the cache's heads, dim]; block_table and seq_lens one row per "
                         "sequence, starts one more")
    held = width * cache.page_size
    if max_len is None:
        max_len = held
    elif not 0 <= max_len <= held:
        raise ValueError("max_len must be within what block_table holds")
    most = T if tree is None else min(T, _TREE_MOST)
    if max_new is None or max_new > T:
        max_new = most
    elif max_new < 0 or max_new > most:
        raise ValueError("max_new must not be negative, nor above 64 in a tree")
    m = None
    if tree is not None or prefix_lens is not None or slopes is not None or window or cap:
        tp = pp = sp = None
        if tree is not None:
            tp = P._vector("tree", tree, P.i64, device)
            if tree.shape[0] != T:
                raise ValueError("tree must have one entry per token")
        if prefix_lens is not None:
            pp = P._vector("prefix_lens", prefix_lens, P.i32, device)
            if prefix_lens.shape[0] != B:
                raise ValueError("prefix_lens must have one entry per sequence")
        if slopes is not None:
            sp = P._vector("slopes", slopes, P.f32, device)
            if slopes.shape[0] != Hq:
                raise ValueError("slopes must have one entry per query head")
        m = _byref(N.QuartzTokensMask(tp, pp, sp, window, cap))
    if out is None:
        out_dtype = out_dtype or q.dtype
        o = P._empty((T, Hq, D), out_dtype, cache.device, stream)
    else:
        o, out_dtype = out, out.dtype
        P._rows("out", o, 3, out_dtype, device)
        if o.shape != q.shape or not o.is_contiguous():
            raise ValueError("out must be contiguous, of the shape of q")
    kind = P._KIND.get(out_dtype)
    if kind is None:
        raise ValueError("the result is float16, bfloat16 or float32")
    if workspace is None:
        size = cache._tokens_workspace_size(T, B, Hq, max_len, max_new)
        workspace = cache._no_workspace if size <= P._NO_WORKSPACE else P._empty((size,), P.torch.uint8, cache.device, stream)
    else:
        if workspace.get_device() != device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA tensor on the current device")
        size = workspace.numel() * workspace.element_size()
    rc = P.lib.quartz_paged_attention_tokens(q.data_ptr(), qs[0], qs[1], T, Hq, cache._ref, block_table.data_ptr(), ts[0],
                                             lens, at, B, max_len, max_new, m, scale, o.data_ptr(), kind,
                                             workspace.data_ptr(), size, _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_paged_attention_tokens")
    return o


def attention_paged_tokens_workspace_size(cache: P.PagedCache, tokens: int, seqs: int, q_heads: int, max_len: int,
                                          max_new: int) -> int:
    return cache._tokens_workspace_size(tokens, seqs, q_heads, max_len, max_new)
