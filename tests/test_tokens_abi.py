"""The entry points for several new tokens per sequence refuse bad arguments on the
host, before anything is launched (no GPU)."""
import ctypes as C
import math

import pytest

from paper_2509_26436_gb300 import _native as N
from paper_2509_26436_gb300 import build as B

torch = pytest.importorskip("torch")
P = 0x10000  # an aligned address that no check dereferences
BAD, ALIGN, UNSUP, WS = (N.QUARTZ_ERR_INVALID_ARG, N.QUARTZ_ERR_ALIGNMENT, N.QUARTZ_ERR_UNSUPPORTED,
                         N.QUARTZ_ERR_WORKSPACE)


@pytest.fixture(scope="module")
def lib():
    B.build()
    return N.load()


def _rope(**kw):
    d = dict(positions=P, axis_stride=64, freqs=P, pair_axis=P, axes=3, rotary=64, interleaved=0, backward=0, scale=1.0)
    d.update(kw)
    return N.QuartzRopeAxes(**d)


ROPE_REFUSALS = [(dict(positions=None), BAD), (dict(freqs=None), BAD), (dict(pair_axis=None), BAD), (dict(axes=0), BAD),
                 (dict(axes=17), BAD), (dict(axis_stride=-1), BAD), (dict(rotary=0), BAD), (dict(rotary=63), BAD),
                 (dict(rotary=130), BAD), (dict(interleaved=2), BAD), (dict(backward=2), BAD), (dict(scale=math.inf), BAD),
                 (dict(scale=math.nan), BAD), (dict(positions=P + 4), ALIGN), (dict(freqs=P + 4), ALIGN),
                 (dict(pair_axis=P + 2), ALIGN)]


def test_rope_axes_refusals(lib):
    def call(x=P, xs=(256, 128), y=P, ys=(256, 128), t=0, T=3, H=2, D=128, r=None):
        return lib.quartz_rope_axes(x, *xs, y, *ys, t, T, H, D, C.byref(r or _rope()), None)

    for kw, status in ROPE_REFUSALS:
        assert call(r=_rope(**kw)) == status, kw
    assert call(t=3) == BAD and call(T=-1) == BAD and call(H=-1) == BAD and call(H=65536) == BAD and call(D=1) == BAD
    assert call(D=320) == UNSUP and call(T=(1 << 30) + 1) == BAD
    assert call(x=None) == BAD and call(y=None) == BAD and call(xs=(-1, 128)) == BAD and call(ys=(256, -128)) == BAD
    assert call(ys=(0, 128)) == BAD and call(ys=(256, 0)) == BAD
    assert call(x=P + 1) == ALIGN and call(t=2, y=P + 2) == ALIGN
    assert lib.quartz_rope_axes(P, 256, 128, P, 256, 128, 0, 3, 2, 128, None, None) == BAD
    assert call(T=0, x=None) == 0 and call(H=0, x=None) == 0


def _side(**kw):
    d = dict(x=P, x_stride_token=256, x_stride_head=128, dy=P, dy_stride_token=256, dy_stride_head=128, y=P,
             y_stride_token=256, y_stride_head=128, w=P, dw=P, heads=2)
    d.update(kw)
    return N.QuartzNormSide(**d)


SIDE_REFUSALS = [(dict(heads=-1), BAD), (dict(heads=65536), BAD), (dict(x=None), BAD), (dict(y=None), BAD),
                 (dict(x_stride_token=-1), BAD), (dict(y_stride_head=-1), BAD), (dict(x_stride_head=1 << 41), BAD),
                 (dict(y_stride_token=0), BAD), (dict(y_stride_head=0), BAD), (dict(x=P + 1), ALIGN), (dict(w=P + 2), ALIGN),
                 (dict(y=P + 1), ALIGN)]
GRAD_REFUSALS = [(dict(dy=None), BAD), (dict(dy_stride_token=-1), BAD), (dict(dy=P + 1), ALIGN), (dict(dw=P + 2), ALIGN)]


@pytest.mark.parametrize("which", ["q", "k"])
def test_norm_refusals(lib, which):
    def call(t=0, wt=2, T=3, D=128, eps=1e-6, r=None, backward=False, ws=P, wsb=1 << 24, **kw):
        sides = [_side(**kw) if which == s else _side() for s in "qk"]
        r = None if r is None else C.byref(r)
        if backward:
            return lib.quartz_qk_norm_rope_backward(C.byref(sides[0]), C.byref(sides[1]), t, wt, T, D, eps, r, ws, wsb, None)
        return lib.quartz_qk_norm_rope(C.byref(sides[0]), C.byref(sides[1]), t, wt, T, D, eps, r, None)

    for backward in (False, True):
        for kw, status in SIDE_REFUSALS:
            assert call(backward=backward, **kw) == status, kw
        for kw, status in ROPE_REFUSALS:
            assert call(backward=backward, r=_rope(**kw)) == status, kw
        assert call(backward=backward, r=_rope(backward=1)) == BAD
        assert call(backward=backward, t=3) == BAD and call(backward=backward, wt=-1) == BAD
        assert call(backward=backward, T=-1) == BAD and call(backward=backward, D=1) == BAD
        assert call(backward=backward, D=320) == UNSUP
        for eps in (-1e-6, math.inf, math.nan):
            assert call(backward=backward, eps=eps) == BAD
    for kw, status in GRAD_REFUSALS:
        assert call(backward=True, **kw) == status, kw
    assert call(backward=True, ws=None) == WS and call(backward=True, wsb=64) == WS and call(backward=True, ws=P + 4) == ALIGN
    assert call(T=0, x=None) == 0
    assert lib.quartz_qk_norm_rope(None, C.byref(_side()), 0, 0, 3, 128, 0.0, None, None) == BAD


def test_workspace_sizes(lib):
    assert lib.quartz_qk_norm_rope_workspace_size(0) == 0 and lib.quartz_qk_norm_rope_workspace_size(512) == 0
    assert lib.quartz_qk_norm_rope_workspace_size(128) >= 128 * 4


@pytest.mark.parametrize("name", ["q", "k", "wq", "wk"])
def test_a_gradient_that_would_be_lost_is_refused(lib, name):
    import paper_2509_26436_gb300 as Q
    t = dict(q=torch.zeros(3, 2, 64), k=torch.zeros(3, 1, 64), wq=torch.ones(64), wk=torch.ones(64))
    t[name].requires_grad_(True)
    with pytest.raises(ValueError, match="records no gradient"):
        Q.qk_norm_rope(t["q"], t["k"], t["wq"], t["wk"])
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):
        Q.qk_norm_rope(t["q"], t["k"], t["wq"], t["wk"])
    x = torch.zeros(3, 2, 64, requires_grad=True)
    with pytest.raises(ValueError, match="records no gradient"):
        Q.rope_axes(x, torch.zeros(2, 3, dtype=torch.int64), torch.ones(32, dtype=torch.float64),
                    torch.zeros(32, dtype=torch.int32))
    with pytest.raises(ValueError, match="records no gradient"):
        Q.qk_norm_rope_backward(x, None, x.detach(), None, None, None)


def _cache(kind=N.PAGES_F16, page=16, heads=2, dim=128, pages=4, data=P):
    side = N.QuartzPages()
    side.data = data
    side.stride_page, side.stride_slot, side.stride_head = page * heads * dim, heads * dim, dim
    return N.QuartzPagedCache(kind, page, heads, dim, pages, side, side)


def test_attention_refusals(lib):
    def call(q=P, qs=(256, 128), T=5, Hq=4, cache=None, table=P, lens=P, starts=P, B=2, max_len=64, max_new=5, scale=1.0,
             o=P, t=0, ws=P, wsb=1 << 40, ts=4, **m):
        mask = C.byref(N.QuartzTokensMask(**m)) if m else None
        return lib.quartz_paged_attention_tokens(q, *qs, T, Hq, C.byref(cache or _cache()), table, ts, lens, starts, B,
                                                 max_len, max_new, mask, scale, o, t, ws, wsb, None)

    assert call(cache=_cache(dim=96)) == UNSUP and call(cache=_cache(data=None)) == BAD and call(cache=_cache(page=24)) == BAD
    assert call(T=-1) == BAD and call(T=(1 << 30) + 1) == BAD and call(B=-1) == BAD and call(B=65536) == BAD
    assert call(Hq=3) == BAD and call(Hq=0) == BAD and call(max_len=-1) == BAD and call(max_len=(1 << 30) + 1) == BAD
    assert call(max_new=-1) == BAD and call(max_new=(1 << 29) + 1) == BAD
    assert call(scale=math.nan) == BAD and call(scale=math.inf) == BAD and call(scale=3e38) == BAD and call(t=3) == BAD
    assert call(window=-1) == BAD and call(cap=-1.0) == BAD and call(cap=math.nan) == BAD and call(cap=3e38) == BAD
    assert call(scale=1e30, cap=1e-30) == BAD and call(tree=P, max_new=65) == BAD
    assert call(tree=P + 4) == ALIGN and call(prefix_lens=P + 2) == ALIGN and call(slopes=P + 2) == ALIGN
    assert call(q=None) == BAD and call(o=None) == BAD and call(lens=None) == BAD and call(starts=None) == BAD
    assert call(table=None) == BAD and call(qs=(-8, 128)) == BAD and call(ts=-1) == BAD
    assert call(q=P + 2) == ALIGN and call(o=P + 4) == ALIGN and call(qs=(252, 128)) == ALIGN and call(qs=(256, 4)) == ALIGN
    assert call(lens=P + 2) == ALIGN and call(starts=P + 2) == ALIGN and call(table=P + 2) == ALIGN
    assert call(ws=None) == WS and call(wsb=0) == WS and call(ws=P + 4) == ALIGN
    assert call(B=0, q=None) == 0 and call(T=0, q=None) == 0 and call(max_new=0, q=None) == 0
    assert lib.quartz_paged_attention_tokens_workspace_size(C.byref(_cache(dim=96)), 5, 2, 4, 64, 5) == 0
    assert lib.quartz_paged_attention_tokens_workspace_size(C.byref(_cache()), 5, 2, 4, 64, 5) > 0
