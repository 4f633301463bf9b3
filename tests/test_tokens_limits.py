"""The largest calls of attention of several new tokens: refused on the host where a
CTA could not count its tiles (no GPU)."""
import ctypes as C

import pytest

from paper_2509_26436_gb300 import _native as N
from test_tokens_abi import P, UNSUP, WS, _cache, lib  # noqa: F401

M = 1 << 20


@pytest.mark.parametrize("T,Hq,heads,dim,ok", [(M, 64, 1, 256, True), (M, 128, 1, 128, True), (4 * M, 8, 1, 128, True),
                                               (8 * M, 64, 8, 128, False), (64 * M, 8, 8, 64, False),
                                               (1 << 30, 1, 1, 64, False)])
def test_tiles_that_a_cta_cannot_count_are_refused(lib, T, Hq, heads, dim, ok):  # noqa: F811
    cache = _cache(page=4096, heads=heads, dim=dim, pages=1 << 18)
    size = lib.quartz_paged_attention_tokens_workspace_size(C.byref(cache), T, 1, Hq, T, T)
    status = lib.quartz_paged_attention_tokens(P, Hq * dim, dim, T, Hq, C.byref(cache), P, 1 << 18, P, P, 1, T, T, None, 1.0,
                                               P, N.OUT_F16, P, 0, None)
    assert (size > 0, status) == ((True, WS) if ok else (False, UNSUP))
