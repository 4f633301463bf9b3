"""Paged key / value cache: rotary positions, the append into pages, attention
of one new token per sequence, and eviction by accumulated attention weight.

As the rest of the package this only marshals torch CUDA tensors into the C
ABI; every call is asynchronous on the current stream (or `stream`).  Autograd
sees none of it: rope(), which training needs too, refuses a tensor whose
gradient would be lost; the others are steps of serving.

    freqs, scale = rope_frequencies(128, base=500000.0, device="cuda")
    cache = empty_paged_cache(num_pages, 64, heads=8, dim=128, params=Params(group_s=16))
    q = rope(q, positions, freqs, scale=scale)
    paged_append(cache, k, v, slots, positions=positions, freqs=freqs, rope_scale=scale)
    o = attention_paged(q, cache, block_table, seq_lens, 128 ** -0.5, weights=weights)
    kept, new_lens = evict_select(weights, seq_lens, budget, recent=256, sinks=4)
    cache_compact(cache, block_table, seq_lens, kept, new_lens, weights=weights)
"""
from __future__ import annotations

import ctypes as C
import math

import paper_2509_26436_gb300 as _Q

from . import _native as N

_byref = C.byref


# torch and its types, bound on the first use (the package is imported without
# torch); lib is the loaded library.
torch = f16 = bf16 = f32 = f64 = i32 = i64 = lib = _device = None
_KIND = {}  # torch type -> quartz_out_t
_NO_WORKSPACE = 256  # attention's workspace where one kernel does all: nothing is written to it


def _bind():
    global torch, f16, bf16, f32, f64, i32, i64, lib, _device
    t = _Q._torch()
    f16, bf16, f32, f64, i32, i64 = t.float16, t.bfloat16, t.float32, t.float64, t.int32, t.int64
    _KIND.update({f16: N.OUT_F16, bf16: N.OUT_BF16, f32: N.OUT_F32})
    _device = getattr(t._C, "_cuda_getDevice", None) or t.cuda.current_device
    lib = N.load()
    torch = t


def _refuse(name, x, dim, kind, last=True):
    """Say what is wrong with x (called where a call's quick check failed)."""
    if not (x.is_cuda and x.dim() == dim and x.dtype is kind and (not last or x.stride(-1) == 1 or x.shape[-1] <= 1)):
        raise ValueError(f"{name} must be a {dim}-D {str(kind).replace('torch.', '')} CUDA tensor" +
                         (" with a contiguous last dimension" if last else ""))
    raise ValueError(f"{name} is on another device than the current one")


def _vector(name, x, kind, device):
    """x is a contiguous 1-D tensor of `kind` on the current device; its address."""
    if not (x.dtype is kind and x.dim() == 1 and x.get_device() == device and (x.is_contiguous())):
        _refuse(name, x, 1, kind)
    return x.data_ptr()


def _rows(name, x, dim, kind, device):
    """x is a `dim`-D tensor of `kind` with a contiguous last dimension on the
    current device; its strides."""
    st = x.stride()
    if not (x.dtype is kind and len(st) == dim and x.get_device() == device and (st[-1] == 1 or x.shape[-1] <= 1)):
        _refuse(name, x, dim, kind)
    return st


def _empty(shape, dtype, device, stream):
    """Uninitialised memory of the stream that the call runs on: memory of
    another one could still be in use there, or be given away too early."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# --- rotary positions ---------------------------------------------------------

def rope_frequencies(rotary: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original_length: int = 8192, beta_fast: float = 32.0, beta_slow: float = 1.0,
                     low_freq_factor: float = 1.0, high_freq_factor: float = 4.0, device="cuda"):
    """Radians per position of each of the rotary / 2 pairs (float64), and the
    factor on cosine and sine: base^(-2 i / rotary), and for long contexts

    scaling "linear": all divided by `factor`;
    "yarn": divided by `factor` below beta_slow turns over `original_length`
        tokens, as they are above beta_fast turns, a ramp over the pairs
        between; cosine and sine times 0.1 ln(factor) + 1;
    "llama3": the same between low_freq_factor and high_freq_factor turns,
        with the ramp over the turns, and no factor."""
    if torch is None:
        import torch as t
    else:
        t = torch
    if rotary < 2 or rotary % 2 or not base > 0 or not factor > 0 or not original_length > 0:
        raise ValueError("rotary must be even and positive; base, factor and original_length positive")
    i = t.arange(rotary // 2, dtype=t.float64)
    f = float(base) ** (-2.0 * i / rotary)
    scale = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "yarn":
        if not (0 < beta_slow < beta_fast and base > 1):
            raise ValueError("0 < beta_slow < beta_fast and base > 1 are needed")
        lo, hi = (rotary * math.log(original_length / (turns * 2 * math.pi)) / (2 * math.log(base))
                  for turns in (beta_fast, beta_slow))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rotary - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f / factor * ramp + f * (1 - ramp)
        scale = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    elif scaling == "llama3":
        if not 0 < low_freq_factor < high_freq_factor:
            raise ValueError("0 < low_freq_factor < high_freq_factor is needed")
        turns = original_length * f / (2 * math.pi)
        keep = ((turns - low_freq_factor) / (high_freq_factor - low_freq_factor)).clamp(0, 1)
        f = (1 - keep) * f / factor + keep * f
    elif scaling != "none":
        raise ValueError('scaling must be "none", "linear", "yarn" or "llama3"')
    return f.to(device), scale


def _rope_struct(positions, freqs, tokens, scale, interleaved, backward, device) -> N.QuartzRope:
    at, f = _vector("positions", positions, i64, device), _vector("freqs", freqs, f64, device)
    if positions.shape[0] != tokens:
        raise ValueError("positions must have one entry per token")
    return N.QuartzRope(at, f, 2 * freqs.shape[0], interleaved, backward, scale)


def rope(x, positions, freqs, interleaved: bool = False, scale: float = 1.0, backward: bool = False, out=None,
         stream=None):
    """x [tokens, heads, dim] (float16, bfloat16 or float32; any strides with a
    contiguous last dimension) with the first 2 len(freqs) elements of each
    head turned by positions[t] * freqs: pairs (i, i + len(freqs)), or
    (2 i, 2 i + 1) with `interleaved`; the rest is copied.  `backward` applies
    the transpose: the gradient of x from that of the result.  `out` may be x
    itself (in place), or must not overlap it.  Nothing is recorded for
    autograd: where gradients are enabled, an x or `out` that requires one is
    refused (call it from an autograd function's forward and, with `backward`,
    from its backward)."""
    if torch is None:
        _bind()
    if (x.requires_grad or (out is not None and out.requires_grad)) and torch.is_grad_enabled():
        raise ValueError("rope records no gradient: use torch.no_grad(), or an autograd function whose backward calls "
                         "rope(..., backward=True)")
    dtype = x.dtype
    kind = _KIND.get(dtype)
    if kind is None or not x.is_cuda:
        raise ValueError("x must be a 3-D float16, bfloat16 or float32 CUDA tensor")
    device = _device()
    xs = _rows("x", x, 3, dtype, device)
    T, H, D = x.shape
    r = _rope_struct(positions, freqs, T, scale, interleaved, backward, device)
    if out is None:
        out = _empty((T, H, D), dtype, x.device, stream)
        s0, s1 = H * D, D
    else:
        s0, s1, _ = _rows("out", out, 3, dtype, device)
        if out.shape != x.shape:
            raise ValueError("out must have the shape of x")
    rc = lib.quartz_rope(x.data_ptr(), xs[0], xs[1], out.data_ptr(), s0, s1, kind, T, H, D, _byref(r), _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_rope")
    return out


# --- the cache ----------------------------------------------------------------

class PagedCache:
    """Keys and values in pages of `page_size` tokens (a power of two).

    16-bit pages: k and v float16 or bfloat16 [pages, page_size, heads, dim]
    (any strides that are multiples of 8, the last dimension contiguous: a
    [pages, heads, page_size, dim] pool goes in as pool.transpose(1, 2)).
    Encoded pages: k and v Encoded with pages * heads * page_size rows of dim
    columns, token (page, head, slot) in row (page * heads + head) * page_size
    + slot; `heads` must then be given.  dim is 64, 128, 192 or 256.

    The object holds the tensors and the description that the calls pass on;
    it is made once and kept as long as the tensors are."""

    def __init__(self, k, v, page_size: int, heads: int | None = None):
        if torch is None:
            _bind()
        self.k, self.v, self.page_size = k, v, page_size
        if page_size < 1 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two")
        if isinstance(k, _Q.Encoded):
            if heads is None or heads < 1 or not isinstance(v, _Q.Encoded) or k.rows != v.rows or k.K != v.K or \
                    k.rows % (heads * page_size):
                raise ValueError("encoded pages need `heads`, and k and v of pages * heads * page_size equal rows")
            for e in (k, v):
                sizes = [(e.codes, 1, e.rows * (e.K // 2)), (e.scales, 2, e.rows * (e.K // 64)),
                         (e.flags, 1, e.rows * (e.K // e.params.group_s))]
                if any(not (t.is_cuda and t.device == k.codes.device and t.is_contiguous() and t.element_size() == width and
                            t.numel() >= n) for t, width, n in sizes):
                    raise ValueError("encoded pages must be contiguous CUDA tensors of one device, of their type and full size")
            self.heads, self.dim, self.num_pages = heads, k.K, k.rows // (heads * page_size)
            self.dtype, self.device = f16, k.codes.device
            sides = [N.QuartzPages(None, 0, 0, 0, e.c()) for e in (k, v)]
            kind = N.PAGES_ENCODED
        else:
            for name, t in (("k", k), ("v", v)):
                if not (t.is_cuda and t.dim() == 4 and t.dtype in (f16, bf16) and t.stride(3) == 1):
                    raise ValueError(f"{name} must be a [pages, page_size, heads, dim] float16 or bfloat16 CUDA tensor "
                                     "with a contiguous last dimension")
            if k.device != v.device:
                raise ValueError("k and v are on different devices")
            if k.shape != v.shape or k.dtype != v.dtype or k.shape[1] != page_size or heads not in (None, k.shape[2]):
                raise ValueError("k and v must agree in shape and type, and have page_size slots and `heads` heads")
            self.num_pages, _, self.heads, self.dim = k.shape
            self.dtype, self.device = k.dtype, k.device
            sides = [N.QuartzPages(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2), N.QuartzEncoded()) for t in (k, v)]
            kind = N.PAGES_F16 if k.dtype is f16 else N.PAGES_BF16
        self.c = N.QuartzPagedCache(kind, page_size, self.heads, self.dim, self.num_pages, *sides)
        self._ref = _byref(self.c)
        self._index = self.device.index
        self._workspace_sizes = {}
        self._no_workspace = torch.empty(_NO_WORKSPACE, dtype=torch.uint8, device=self.device)

    def _workspace_size(self, seqs, q_heads, max_len, window, with_weights) -> int:
        key = (seqs, q_heads, max_len, window, with_weights)
        n = self._workspace_sizes.get(key)
        if n is None:
            if len(self._workspace_sizes) >= 1024:
                self._workspace_sizes.clear()
            n = N.load().quartz_paged_attention_workspace_size(self._ref, seqs, q_heads, max_len, window, with_weights)
            self._workspace_sizes[key] = n
        return n

    def _check_device(self) -> int:
        device = _device()
        if self._index != device:
            raise ValueError("the cache is on another device than the current one")
        return device


def empty_paged_cache(num_pages: int, page_size: int, heads: int, dim: int, dtype=None, params=None,
                      device="cuda") -> PagedCache:
    """A cache with uninitialised pages: 16-bit ones of `dtype` (float16 by
    default), or encoded ones of `params`."""
    if torch is None:
        _bind()
    if params is not None:
        k, v = (_Q.empty_encoded(num_pages * heads * page_size, dim, params, device) for _ in range(2))
        return PagedCache(k, v, page_size, heads)
    k, v = (torch.empty((num_pages, page_size, heads, dim), dtype=dtype or torch.float16, device=device)
            for _ in range(2))
    return PagedCache(k, v, page_size)


def paged_append(cache: PagedCache, k, v, slots, positions=None, freqs=None, interleaved: bool = False,
                 rope_scale: float = 1.0, stream=None) -> None:
    """Write k and v [tokens, heads, dim] (the cache's type; float16 for encoded
    pages, which store Eq. 1 + Eq. 2 of them) to slots[t] = page * page_size +
    slot (int64; negative ones are skipped, no two are alike).  With
    `positions` and `freqs` the keys are rotated on the way, as rope() does."""
    device, kind = cache._check_device(), cache.dtype
    ks, vs = _rows("k", k, 3, kind, device), _rows("v", v, 3, kind, device)
    at = _vector("slots", slots, i64, device)
    T = slots.shape[0]
    if k.shape != (T, cache.heads, cache.dim) or v.shape != k.shape:
        raise ValueError("k and v must be [tokens, heads, dim] of the cache, with one slot per token")
    r = None
    if positions is not None and freqs is not None:
        r = _byref(_rope_struct(positions, freqs, T, rope_scale, interleaved, False, device))
    elif positions is not None or freqs is not None:
        raise ValueError("positions and freqs go together")
    rc = lib.quartz_paged_append(cache._ref, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], T, at, r,
                                 _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_paged_append")


def attention_paged(q, cache: PagedCache, block_table, seq_lens, scale: float, window: int = 0,
                    max_len: int | None = None, out_dtype=None, out=None, weights=None, workspace=None, stream=None):
    """o [seqs, q_heads, dim]: one new query per sequence over its cached tokens
    (the last `window` of them if window > 0).  q [seqs, q_heads, dim] in the
    cache's type (float16 for encoded pages); block_table int32 [seqs, pages];
    seq_lens int32 [seqs], at most max_len (default: what the table holds; a
    smaller known bound plans fewer splits).  weights float32 [seqs, heads, >=
    max_len]: the attention weights, summed over each head's queries, are added
    in place.  A workspace of the caller's is only good for one call at a time,
    and for one captured graph."""
    device = cache._check_device()
    qs = _rows("q", q, 3, cache.dtype, device)
    ts = _rows("block_table", block_table, 2, i32, device)
    lens = _vector("seq_lens", seq_lens, i32, device)
    B, Hq, D = q.shape
    n, width = block_table.shape
    if D != cache.dim or Hq % cache.heads or n != B or seq_lens.shape[0] != B:
        raise ValueError("q must be [seqs, a multiple of the cache's heads, dim]; block_table and seq_lens one row per sequence")
    held = width * cache.page_size
    if max_len is None:
        max_len = held
    elif not 0 <= max_len <= held:
        raise ValueError("max_len must be within what block_table holds")
    if out is None:
        out_dtype = out_dtype or q.dtype
        o = _empty((B, Hq, D), out_dtype, cache.device, stream)
    else:
        o, out_dtype = out, out.dtype
        _rows("out", o, 3, out_dtype, device)
        if o.shape != q.shape or not o.is_contiguous():
            raise ValueError("out must be contiguous, of the shape of q")
    kind = _KIND.get(out_dtype)
    if kind is None:
        raise ValueError("the result is float16, bfloat16 or float32")
    w_ptr, w_sb, w_sh, with_weights = None, 0, 0, 0
    if weights is not None:
        w_sb, w_sh, _ = _rows("weights", weights, 3, f32, device)
        if weights.shape[0] != B or weights.shape[1] != cache.heads or weights.shape[2] < max_len:
            raise ValueError("weights must be [seqs, heads, at least max_len]")
        w_ptr, with_weights = weights.data_ptr(), 1
    if workspace is None:
        size = cache._workspace_size(B, Hq, max_len, window, with_weights)
        workspace = cache._no_workspace if size <= _NO_WORKSPACE else _empty(size, torch.uint8, cache.device, stream)
    else:
        if workspace.get_device() != device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA tensor on the current device")
        size = workspace.numel() * workspace.element_size()
    rc = lib.quartz_paged_attention(q.data_ptr(), qs[0], qs[1], B, Hq, cache._ref, block_table.data_ptr(), ts[0], lens,
                                    max_len, window, scale, o.data_ptr(), kind, w_ptr, w_sb, w_sh, workspace.data_ptr(),
                                    size, _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_paged_attention")
    return o


def attention_paged_workspace_size(cache: PagedCache, seqs: int, q_heads: int, max_len: int, window: int = 0,
                                   with_weights: bool = False) -> int:
    return cache._workspace_size(seqs, q_heads, max_len, window, 1 if with_weights else 0)


def evict_select(weights, seq_lens, budget: int, recent: int = 0, sinks: int = 0, max_len: int | None = None, kept=None,
                 new_lens=None, stream=None):
    """(kept int32 [seqs, heads, budget], new_lens int32 [seqs]): the tokens
    that stay in each head's cache, ascending and then -1: all of them up to
    `budget`, else the first `sinks`, the last `recent` and the largest
    weights between (ties: the lowest index; NaN is the smallest).  `new_lens`
    must not be seq_lens, which cache_compact needs too."""
    if torch is None:
        _bind()
    if not weights.is_cuda:
        _refuse("weights", weights, 3, f32)
    device = _device()
    sb, sh, _ = _rows("weights", weights, 3, f32, device)
    lens = _vector("seq_lens", seq_lens, i32, device)
    B, H, n = weights.shape
    if seq_lens.shape[0] != B:
        raise ValueError("seq_lens must have one entry per sequence")
    if max_len is None:
        max_len = n
    elif not 0 <= max_len <= n:
        raise ValueError("max_len must be within weights' last dimension")
    if kept is None:
        kept = _empty((B, H, max(budget, 0)), i32, weights.device, stream)
    else:
        _rows("kept", kept, 3, i32, device)
        if kept.shape != (B, H, budget) or not kept.is_contiguous():
            raise ValueError("kept must be contiguous [seqs, heads, budget]")
    if new_lens is None:
        new_lens = _empty((B,), i32, weights.device, stream)
    elif new_lens.shape[0] != B:
        raise ValueError("new_lens must have one entry per sequence")
    rc = lib.quartz_evict_select(weights.data_ptr(), sb, sh, lens, B, H, max_len, budget, recent, sinks, kept.data_ptr(),
                                 _vector("new_lens", new_lens, i32, device), _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_evict_select")
    return kept, new_lens


def cache_compact(cache: PagedCache, block_table, seq_lens, kept, new_lens=None, new_table=None, weights=None,
                  max_len: int | None = None, stream=None) -> None:
    """Close up the cache: row j of every sequence and head becomes its row
    kept[b, h, j], j < min(len, budget) (= new_lens, which is not needed again).
    In place in block_table's pages (then one sequence's each), or into the
    pages of new_table, which are none of block_table's.  `weights` (the sums
    of attention_paged) close up in place alike, with 0 from the new length to
    the old."""
    device = cache._check_device()
    ts = _rows("block_table", block_table, 2, i32, device)
    lens = _vector("seq_lens", seq_lens, i32, device)
    _rows("kept", kept, 3, i32, device)
    B, H, budget = kept.shape
    n, width = block_table.shape
    if H != cache.heads or n != B or seq_lens.shape[0] != B or not kept.is_contiguous():
        raise ValueError("kept must be contiguous [seqs, heads, budget]; block_table and seq_lens one row per sequence")
    held = width * cache.page_size
    if max_len is None:
        max_len = held
    elif not 0 <= max_len <= held:
        raise ValueError("max_len must be within what block_table holds")
    n_ptr, n_stride = None, 0
    if new_table is not None:
        n_stride = _rows("new_table", new_table, 2, i32, device)[0]
        if new_table.shape[0] != B or new_table.shape[1] * cache.page_size < min(budget, max_len):
            raise ValueError("new_table must hold min(budget, max_len) tokens of each sequence")
        n_ptr = new_table.data_ptr()
    w_ptr, w_sb, w_sh = None, 0, 0
    if weights is not None:
        w_sb, w_sh, _ = _rows("weights", weights, 3, f32, device)
        if weights.shape[0] != B or weights.shape[1] != H or weights.shape[2] < max_len:
            raise ValueError("weights must be [seqs, heads, at least max_len]")
        w_ptr = weights.data_ptr()
    rc = lib.quartz_cache_compact(cache._ref, B, block_table.data_ptr(), ts[0], n_ptr, n_stride, lens, max_len,
                                  kept.data_ptr(), budget, w_ptr, w_sb, w_sh, _Q._stream(stream))
    if rc:
        N.check(rc, "quartz_cache_compact")
