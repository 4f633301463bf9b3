"""The paged cache's entry points refuse bad arguments on the host, before
anything is launched (no GPU), and the frequencies are the formulas'."""
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
    d = dict(positions=P, freqs=P, rotary=64, interleaved=0, backward=0, scale=1.0)
    d.update(kw)
    return N.QuartzRope(**d)


def _cache(kind=N.PAGES_F16, page=16, heads=2, dim=128, pages=4, gs=16, flag_bits=8, code_bits=8, mode=0, rows=None,
           data=P, strides=None):
    side = N.QuartzPages()
    if kind == N.PAGES_ENCODED:
        rows = pages * heads * page if rows is None else rows
        side.enc = N.QuartzEncoded(data, data, data, None, None, rows, dim, N.QuartzParams(64, gs, mode, flag_bits, code_bits))
    else:
        side.data = data
        side.stride_page, side.stride_slot, side.stride_head = strides or (page * heads * dim, heads * dim, dim)
    return N.QuartzPagedCache(kind, page, heads, dim, pages, side, side)


def test_rope_refusals(lib):
    def call(x=P, xs=(256, 128), y=P, ys=(256, 128), t=0, T=3, H=2, D=128, r=None):
        r = r or _rope()
        return lib.quartz_rope(x, *xs, y, *ys, t, T, H, D, C.byref(r), None)

    assert call(t=3) == BAD and call(T=-1) == BAD and call(H=-1) == BAD and call(D=1) == BAD and call(D=2048) == BAD
    assert call(x=None) == BAD and call(y=None) == BAD
    assert call(xs=(-1, 128)) == BAD
    for kw in (dict(positions=None), dict(freqs=None), dict(rotary=0), dict(rotary=63), dict(rotary=130),
               dict(interleaved=2), dict(backward=-1), dict(scale=math.inf), dict(scale=math.nan)):
        assert call(r=_rope(**kw)) == BAD, kw
    assert call(r=_rope(rotary=514), D=1024) == BAD
    assert call(x=P + 1) == ALIGN and call(t=2, y=P + 2) == ALIGN
    assert call(r=_rope(positions=P + 4)) == ALIGN
    assert lib.quartz_rope(P, 0, 0, P, 0, 0, 0, 3, 2, 128, None, None) == BAD
    assert call(T=0, x=None) == 0 and call(H=0) == 0


CACHE_REFUSALS = [(dict(kind=7), BAD), (dict(page=24), BAD), (dict(page=0), BAD), (dict(page=8192), BAD),
                  (dict(heads=0), BAD), (dict(heads=2000), BAD), (dict(pages=0), BAD), (dict(dim=0), BAD),
                  (dict(dim=96), UNSUP), (dict(data=None), BAD), (dict(data=P + 8), ALIGN),
                  (dict(strides=(4096, 2048, -128)), BAD), (dict(strides=(4096, 4, 128)), ALIGN),
                  (dict(strides=(1 << 31, 256, 128)), BAD), (dict(kind=N.PAGES_ENCODED, gs=12), BAD),
                  (dict(kind=N.PAGES_ENCODED, flag_bits=4), UNSUP), (dict(kind=N.PAGES_ENCODED, code_bits=16), UNSUP),
                  (dict(kind=N.PAGES_ENCODED, mode=1), UNSUP), (dict(kind=N.PAGES_ENCODED, rows=127), BAD),
                  (dict(kind=N.PAGES_ENCODED, data=None), BAD), (dict(kind=N.PAGES_ENCODED, data=P + 8), ALIGN),
                  (dict(kind=N.PAGES_ENCODED, pages=1 << 27), UNSUP)]


@pytest.mark.parametrize("kw,status", CACHE_REFUSALS)
def test_cache_refusals(lib, kw, status):
    c = _cache(**kw)
    assert lib.quartz_paged_append(C.byref(c), P, 256, 128, P, 256, 128, 1, P, None, None) == status
    assert lib.quartz_paged_attention_workspace_size(C.byref(c), 1, 2, 64, 0, 0) == 0
    assert lib.quartz_paged_attention(P, 256, 128, 1, 2, C.byref(c), P, 4, P, 64, 0, 1.0, P, 0, None, 0, 0, P, 1 << 30,
                                      None) == status
    assert lib.quartz_cache_compact(C.byref(c), 1, P, 4, None, 0, P, 64, P, 8, None, 0, 0, None) == status


def test_sides_must_agree(lib):
    c = _cache(N.PAGES_ENCODED)
    c.v.enc.p.group_s = 32
    assert lib.quartz_paged_append(C.byref(c), P, 256, 128, P, 256, 128, 1, P, None, None) == BAD


def test_append_refusals(lib):
    c = _cache()

    def call(k=P, ks=(256, 128), v=P, vs=(256, 128), T=1, slots=P, r=None):
        return lib.quartz_paged_append(C.byref(c), k, *ks, v, *vs, T, slots, None if r is None else C.byref(r), None)

    assert lib.quartz_paged_append(None, P, 256, 128, P, 256, 128, 1, P, None, None) == BAD
    assert call(k=None) == BAD and call(v=None) == BAD and call(slots=None) == BAD and call(T=-1) == BAD
    assert call(k=P + 2) == ALIGN and call(v=P + 8) == ALIGN and call(slots=P + 4) == ALIGN
    assert call(ks=(250, 128)) == ALIGN and call(vs=(256, -8)) == BAD
    assert call(r=_rope(rotary=192)) == BAD and call(r=_rope(backward=1)) == BAD
    assert call(T=0, k=None) == 0


def test_attention_refusals(lib):
    c = _cache()

    def call(q=P, qs=(256, 128), B=1, Hq=4, cache=c, table=P, lens=P, max_len=64, window=0, scale=1.0, o=P, t=0, w=None,
             ws=P, wsb=1 << 30, w_st=(0, 0)):
        return lib.quartz_paged_attention(q, *qs, B, Hq, C.byref(cache), table, 4, lens, max_len, window, scale, o, t, w,
                                          *w_st, ws, wsb, None)

    assert call(B=-1) == BAD and call(B=65536) == BAD and call(Hq=3) == BAD and call(Hq=0) == BAD
    assert call(max_len=-1) == BAD and call(max_len=(1 << 30) + 1) == BAD and call(window=-1) == BAD
    assert call(scale=math.nan) == BAD and call(scale=math.inf) == BAD and call(t=5) == BAD
    assert call(q=None) == BAD and call(table=None) == BAD and call(lens=None) == BAD and call(o=None) == BAD
    assert call(q=P + 2) == ALIGN and call(o=P + 4) == ALIGN and call(qs=(252, 128)) == ALIGN and call(w=P + 2) == ALIGN
    assert call(qs=(-8, 128)) == BAD and call(w=P, w_st=(-1, 0)) == BAD
    assert call(ws=None) == WS and call(wsb=0) == WS and call(ws=P + 4) == ALIGN
    assert call(B=0, q=None) == 0


def test_workspace_of_nothing(lib):
    """No sequences, or a table without a place: planned, not divided by."""
    c = _cache()
    for B, n, window in ((0, 64, 0), (1, 0, 0), (0, 0, 0), (1, 64, (1 << 63) - 1), (65535, 1 << 30, 1)):
        for weights in (0, 1):
            assert lib.quartz_paged_attention_workspace_size(C.byref(c), B, 2, n, window, weights) > 0
    assert lib.quartz_paged_attention(None, 256, 128, 0, 2, C.byref(c), None, 0, None, 0, 0, 1.0, None, 0, None, 0, 0, None,
                                      0, None) == 0


def test_token_limits(lib):
    c, r = _cache(), _rope()
    assert lib.quartz_paged_append(C.byref(c), P, 256, 128, P, 256, 128, (1 << 30) + 1, P, None, None) == BAD
    assert lib.quartz_rope(P, 256, 128, P, 256, 128, 0, (1 << 30) + 1, 2, 128, C.byref(r), None) == BAD


def test_evict_refusals(lib):
    def call(w=P, st=(64, 32), lens=P, B=1, H=2, n=32, budget=8, recent=2, sinks=1, kept=P, new=P):
        return lib.quartz_evict_select(w, *st, lens, B, H, n, budget, recent, sinks, kept, new, None)

    for kw in (dict(w=None), dict(lens=None), dict(kept=None), dict(new=None), dict(B=-1), dict(H=0), dict(n=-1),
               dict(budget=0), dict(recent=-1), dict(sinks=-1), dict(recent=8), dict(recent=9, sinks=0),
               dict(budget=(1 << 30) + 1), dict(st=(-1, 0))):
        assert call(**kw) == BAD, kw
    for kw in (dict(w=P + 2), dict(lens=P + 1), dict(kept=P + 2), dict(new=P + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0, w=None) == 0


def test_compact_refusals(lib):
    c = _cache()

    def call(B=1, table=P, st=4, new=None, nst=0, lens=P, n=64, kept=P, budget=8, w=None, ws=(0, 0)):
        return lib.quartz_cache_compact(C.byref(c), B, table, st, new, nst, lens, n, kept, budget, w, *ws, None)

    for kw in (dict(B=-1), dict(table=None), dict(lens=None), dict(kept=None), dict(budget=0), dict(n=-1), dict(st=-1),
               dict(nst=-1), dict(w=P, ws=(0, -1))):
        assert call(**kw) == BAD, kw
    for kw in (dict(table=P + 2), dict(new=P + 2), dict(lens=P + 2), dict(kept=P + 2), dict(w=P + 1)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0) == 0 and call(n=0) == 0


def test_index_status_has_a_name(lib):
    assert lib.quartz_status_string(N.QUARTZ_ERR_INDEX) == b"QUARTZ_ERR_INDEX"


def test_python_checks_need_no_gpu():
    import paper_2509_26436_gb300 as Q
    x = torch.zeros(3, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        Q.rope(x, torch.zeros(3, dtype=torch.int64), torch.ones(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        Q.PagedCache(torch.zeros(2, 16, 2, 64, dtype=torch.float16), torch.zeros(2, 16, 2, 64, dtype=torch.float16), 16)
    with pytest.raises(ValueError):
        Q.evict_select(torch.zeros(1, 2, 8), torch.zeros(1, dtype=torch.int32), 4)


def test_frequencies():
    import paper_2509_26436_gb300 as Q
    f, m = Q.rope_frequencies(8, base=10000.0, device="cpu")
    assert f.dtype == torch.float64 and m == 1.0
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15, atol=0)
    g, m = Q.rope_frequencies(8, base=10000.0, scaling="linear", factor=4.0, device="cpu")
    assert torch.equal(g, f / 4) and m == 1.0
    # llama3: 8192 positions; f = 1, 0.1 make over 4 turns, 0.001 (1.3) is between, 0.0001 under one
    f, _ = Q.rope_frequencies(10, base=100000.0, device="cpu")
    g, m = Q.rope_frequencies(10, base=100000.0, scaling="llama3", factor=8.0, device="cpu")
    assert m == 1.0 and torch.equal(g[:3], f[:3]) and g[4] == f[4] / 8
    keep = (8192 * f[3].item() / (2 * math.pi) - 1) / 3
    assert g[3].item() == pytest.approx((1 - keep) * f[3].item() / 8 + keep * f[3].item(), rel=1e-14)
    g, m = Q.rope_frequencies(64, base=500000.0, scaling="yarn", factor=8.0, device="cpu")
    f, _ = Q.rope_frequencies(64, base=500000.0, device="cpu")
    assert m == pytest.approx(0.1 * math.log(8) + 1) and torch.equal(g[:4], f[:4])
    assert torch.allclose(g[-1], f[-1] / 8, rtol=1e-15, atol=0) and bool((g <= f).all()) and bool((g >= f / 8 * (1 - 1e-15)).all())
    for bad in (dict(rotary=7), dict(rotary=8, scaling="x"), dict(rotary=8, factor=0.0),
                dict(rotary=8, scaling="yarn", beta_fast=1.0, beta_slow=2.0),
                dict(rotary=8, scaling="llama3", low_freq_factor=4.0, high_freq_factor=4.0)):
        with pytest.raises(ValueError):
            Q.rope_frequencies(device="cpu", **bad)
