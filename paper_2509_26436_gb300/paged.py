"""Paged key / value cache: rotary positions, the append into pages, attention
of one new token per sequence, and eviction by accumulated attention weight.

As the rest of the package this only marshals torch CUDA tensors into the C
ABI; every call is asynchronous on the current stream (or `stream`).

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


def _dtypes():
    """(float16, bfloat16, float32, float64, int32, int64)"""
    t = _Q._torch()
    return t.float16, t.bfloat16, t.float32, t.float64, t.int32, t.int64


def _check(name, x, dim, dtypes, last_contiguous=True):
    """x is a `dim`-D CUDA tensor of one of `dtypes` on the current device."""
    if not (x.is_cuda and x.dim() == dim and x.dtype in dtypes and (not last_contiguous or x.stride(-1) == 1 or x.shape[-1] == 1)):
        kinds = " or ".join(str(d).replace("torch.", "") for d in dtypes)
        raise ValueError(f"{name} must be a {dim}-D {kinds} CUDA tensor" +
                         (" with a contiguous last dimension" if last_contiguous else ""))
    if x.get_device() != _current_device():
        raise ValueError(f"{name} is on another device than the current one")


_device_getter = None


def _current_device() -> int:
    global _device_getter
    if _device_getter is None:
        torch = _Q._torch()
        _device_getter = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _device_getter()


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
    torch = _Q._torch()
    if rotary < 2 or rotary % 2 or not base > 0 or not factor > 0 or not original_length > 0:
        raise ValueError("rotary must be even and positive; base, factor and original_length positive")
    i = torch.arange(rotary // 2, dtype=torch.float64)
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


def _rope_struct(positions, freqs, tokens, scale, interleaved, backward) -> N.QuartzRope:
    _, _, _, f64, _, i64 = _dtypes()
    _check("positions", positions, 1, (i64,))
    _check("freqs", freqs, 1, (f64,))
    if positions.shape[0] != tokens:
        raise ValueError("positions must have one entry per token")
    return N.QuartzRope(positions.data_ptr(), freqs.data_ptr(), 2 * freqs.shape[0], int(interleaved), int(backward), scale)


def rope(x, positions, freqs, interleaved: bool = False, scale: float = 1.0, backward: bool = False, out=None,
         stream=None):
    """x [tokens, heads, dim] (float16, bfloat16 or float32; any strides with a
    contiguous last dimension) with the first 2 len(freqs) elements of each
    head turned by positions[t] * freqs: pairs (i, i + len(freqs)), or
    (2 i, 2 i + 1) with `interleaved`; the rest is copied.  `backward` applies
    the transpose: the gradient of x from that of the result.  `out` may be x
    itself (in place), or must not overlap it."""
    f16, bf16, f32, _, _, _ = _dtypes()
    _check("x", x, 3, (f16, bf16, f32))
    T, H, D = x.shape
    if out is None:
        out = _Q._torch().empty((T, H, D), dtype=x.dtype, device=x.device)
    else:
        _check("out", out, 3, (x.dtype,))
        if out.shape != x.shape:
            raise ValueError("out must have the shape of x")
    r = _rope_struct(positions, freqs, T, scale, interleaved, backward)
    xs, os_ = x.stride(), out.stride()
    N.check(N.load().quartz_rope(x.data_ptr(), xs[0], xs[1], out.data_ptr(), os_[0], os_[1], _Q._out_type(x.dtype), T, H,
                                 D, _byref(r), _Q._stream(stream)), "quartz_rope")
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
        f16, bf16, _, _, _, _ = _dtypes()
        self.k, self.v, self.page_size = k, v, page_size
        if page_size < 1 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two")
        if isinstance(k, _Q.Encoded):
            if heads is None or heads < 1 or not isinstance(v, _Q.Encoded) or k.rows != v.rows or k.K != v.K or \
                    k.rows % (heads * page_size):
                raise ValueError("encoded pages need `heads`, and k and v of pages * heads * page_size equal rows")
            for e in (k, v):
                sizes = [(e.codes, e.rows * (e.K // 2)), (e.scales, e.rows * (e.K // 64)),
                         (e.flags, e.rows * (e.K // e.params.group_s))]
                if any(not (t.is_cuda and t.is_contiguous() and t.numel() >= n) for t, n in sizes):
                    raise ValueError("encoded pages must be contiguous CUDA tensors of their full size")
            self.heads, self.dim, self.num_pages = heads, k.K, k.rows // (heads * page_size)
            self.dtype, self.device = f16, k.codes.device
            sides = [N.QuartzPages(None, 0, 0, 0, e.c()) for e in (k, v)]
            kind = N.PAGES_ENCODED
        else:
            for name, t in (("k", k), ("v", v)):
                if not (t.is_cuda and t.dim() == 4 and t.dtype in (f16, bf16) and t.stride(3) == 1):
                    raise ValueError(f"{name} must be a [pages, page_size, heads, dim] float16 or bfloat16 CUDA tensor "
                                     "with a contiguous last dimension")
            if k.shape != v.shape or k.dtype != v.dtype or k.shape[1] != page_size or heads not in (None, k.shape[2]):
                raise ValueError("k and v must agree in shape and type, and have page_size slots and `heads` heads")
            self.num_pages, _, self.heads, self.dim = k.shape
            self.dtype, self.device = k.dtype, k.device
            sides = [N.QuartzPages(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2), N.QuartzEncoded()) for t in (k, v)]
            kind = N.PAGES_F16 if k.dtype is f16 else N.PAGES_BF16
        self.c = N.QuartzPagedCache(kind, page_size, self.heads, self.dim, self.num_pages, *sides)
        self._workspace_sizes = {}

    def _workspace_size(self, seqs, q_heads, max_len, window, with_weights) -> int:
        key = (seqs, q_heads, max_len, window, with_weights)
        n = self._workspace_sizes.get(key)
        if n is None:
            if len(self._workspace_sizes) >= 1024:
                self._workspace_sizes.clear()
            n = N.load().quartz_paged_attention_workspace_size(_byref(self.c), seqs, q_heads, max_len, window, with_weights)
            self._workspace_sizes[key] = n
        return n

    def _check_device(self):
        if self.device.index != _current_device():
            raise ValueError("the cache is on another device than the current one")


def empty_paged_cache(num_pages: int, page_size: int, heads: int, dim: int, dtype=None, params=None,
                      device="cuda") -> PagedCache:
    """A cache with uninitialised pages: 16-bit ones of `dtype` (float16 by
    default), or encoded ones of `params`."""
    torch = _Q._torch()
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
    _, _, _, _, _, i64 = _dtypes()
    _check("k", k, 3, (cache.dtype,))
    _check("v", v, 3, (cache.dtype,))
    _check("slots", slots, 1, (i64,))
    cache._check_device()
    T = slots.shape[0]
    if k.shape != (T, cache.heads, cache.dim) or v.shape != k.shape:
        raise ValueError("k and v must be [tokens, heads, dim] of the cache, with one slot per token")
    if (positions is None) != (freqs is None):
        raise ValueError("positions and freqs go together")
    r = None if freqs is None else _rope_struct(positions, freqs, T, rope_scale, interleaved, False)
    ks, vs = k.stride(), v.stride()
    N.check(N.load().quartz_paged_append(_byref(cache.c), k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], T,
                                         slots.data_ptr(), None if r is None else _byref(r), _Q._stream(stream)),
            "quartz_paged_append")


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
    f16, bf16, f32, _, i32, _ = _dtypes()
    _check("q", q, 3, (cache.dtype,))
    _check("block_table", block_table, 2, (i32,))
    _check("seq_lens", seq_lens, 1, (i32,))
    cache._check_device()
    B, Hq, D = q.shape
    if D != cache.dim or Hq % cache.heads or block_table.shape[0] != B or seq_lens.shape[0] != B:
        raise ValueError("q must be [seqs, a multiple of the cache's heads, dim]; block_table and seq_lens one row per sequence")
    held = block_table.shape[1] * cache.page_size
    if max_len is None:
        max_len = held
    elif not 0 <= max_len <= held:
        raise ValueError("max_len must be within what block_table holds")
    o = out if out is not None else _Q._torch().empty((B, Hq, D), dtype=out_dtype or q.dtype, device=q.device)
    if out is not None:
        _check("out", out, 3, (f16, bf16, f32))
        if out.shape != q.shape or not out.is_contiguous():
            raise ValueError("out must be contiguous, of the shape of q")
    w_ptr, w_sb, w_sh = None, 0, 0
    if weights is not None:
        _check("weights", weights, 3, (f32,))
        if weights.shape[0] != B or weights.shape[1] != cache.heads or weights.shape[2] < max_len:
            raise ValueError("weights must be [seqs, heads, at least max_len]")
        w_ptr, (w_sb, w_sh, _) = weights.data_ptr(), weights.stride()
    need = cache._workspace_size(B, Hq, max_len, window, 1 if weights is not None else 0)
    if workspace is None:
        workspace = _Q._torch().empty(max(need, 16), dtype=_Q._torch().uint8, device=q.device)
    qs = q.stride()
    N.check(N.load().quartz_paged_attention(
        q.data_ptr(), qs[0], qs[1], B, Hq, _byref(cache.c), block_table.data_ptr(), block_table.stride(0),
        seq_lens.data_ptr(), max_len, window, scale, o.data_ptr(), _Q._out_type(o.dtype), w_ptr, w_sb, w_sh,
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), _Q._stream(stream)), "quartz_paged_attention")
    return o


def attention_paged_workspace_size(cache: PagedCache, seqs: int, q_heads: int, max_len: int, window: int = 0,
                                   with_weights: bool = False) -> int:
    return cache._workspace_size(seqs, q_heads, max_len, window, 1 if with_weights else 0)


def evict_select(weights, seq_lens, budget: int, recent: int = 0, sinks: int = 0, max_len: int | None = None, kept=None,
                 new_lens=None, stream=None):
    """(kept int32 [seqs, heads, budget], new_lens int32 [seqs]): the tokens
    that stay in each head's cache, ascending and then -1: all of them up to
    `budget`, else the first `sinks`, the last `recent` and the largest
    weights between (ties: the lowest index; NaN is the smallest)."""
    _, _, f32, _, i32, _ = _dtypes()
    _check("weights", weights, 3, (f32,))
    _check("seq_lens", seq_lens, 1, (i32,))
    B, H, n = weights.shape
    if seq_lens.shape[0] != B:
        raise ValueError("seq_lens must have one entry per sequence")
    if max_len is None:
        max_len = n
    elif not 0 <= max_len <= n:
        raise ValueError("max_len must be within weights' last dimension")
    torch = _Q._torch()
    if kept is None:
        kept = torch.empty((B, H, budget), dtype=torch.int32, device=weights.device)
    if new_lens is None:
        new_lens = torch.empty((B,), dtype=torch.int32, device=weights.device)
    _check("kept", kept, 3, (i32,))
    _check("new_lens", new_lens, 1, (i32,))
    if kept.shape != (B, H, budget) or not kept.is_contiguous() or new_lens.shape[0] != B:
        raise ValueError("kept must be contiguous [seqs, heads, budget], new_lens [seqs]")
    sb, sh, _ = weights.stride()
    N.check(N.load().quartz_evict_select(weights.data_ptr(), sb, sh, seq_lens.data_ptr(), B, H, max_len, budget, recent,
                                         sinks, kept.data_ptr(), new_lens.data_ptr(), _Q._stream(stream)),
            "quartz_evict_select")
    return kept, new_lens


def cache_compact(cache: PagedCache, block_table, seq_lens, kept, new_lens=None, new_table=None, weights=None,
                  max_len: int | None = None, stream=None) -> None:
    """Close up the cache: row j of every sequence and head becomes its row
    kept[b, h, j], j < min(len, budget) (= new_lens, which is not needed again).
    In place in block_table's pages (then one sequence's each), or into the
    pages of new_table, which are none of block_table's.  `weights` (the sums
    of attention_paged) close up in place alike, with 0 from the new length to
    the old."""
    _, _, f32, _, i32, _ = _dtypes()
    _check("block_table", block_table, 2, (i32,))
    _check("seq_lens", seq_lens, 1, (i32,))
    _check("kept", kept, 3, (i32,))
    cache._check_device()
    B, H, budget = kept.shape
    if H != cache.heads or block_table.shape[0] != B or seq_lens.shape[0] != B or not kept.is_contiguous():
        raise ValueError("kept must be contiguous [seqs, heads, budget]; block_table and seq_lens one row per sequence")
    held = block_table.shape[1] * cache.page_size
    if max_len is None:
        max_len = held
    elif not 0 <= max_len <= held:
        raise ValueError("max_len must be within what block_table holds")
    n_ptr, n_stride = None, 0
    if new_table is not None:
        _check("new_table", new_table, 2, (i32,))
        if new_table.shape[0] != B or new_table.shape[1] * cache.page_size < min(budget, max_len):
            raise ValueError("new_table must hold min(budget, max_len) tokens of each sequence")
        n_ptr, n_stride = new_table.data_ptr(), new_table.stride(0)
    w_ptr, w_sb, w_sh = None, 0, 0
    if weights is not None:
        _check("weights", weights, 3, (f32,))
        if weights.shape[0] != B or weights.shape[1] != H or weights.shape[2] < max_len:
            raise ValueError("weights must be [seqs, heads, at least max_len]")
        w_ptr, (w_sb, w_sh, _) = weights.data_ptr(), weights.stride()
    N.check(N.load().quartz_cache_compact(_byref(cache.c), B, block_table.data_ptr(), block_table.stride(0), n_ptr,
                                          n_stride, seq_lens.data_ptr(), max_len, kept.data_ptr(), budget, w_ptr, w_sb,
                                          w_sh, _Q._stream(stream)), "quartz_cache_compact")
