"""Strides of 0 where something is written, so that several elements share a
place: refused.  Read ones are taken."""
import ctypes as C

import pytest

from paper_2509_26436_gb300 import _native as N
from paper_2509_26436_gb300 import build as B

P = 0x10000  # an aligned address that no check dereferences
BAD, WS = N.QUARTZ_ERR_INVALID_ARG, N.QUARTZ_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    B.build()
    return N.load()


def _cache(k=(4096, 256, 128), v=(4096, 256, 128), page=16, heads=2, pages=4):
    sides = []
    for st in (k, v):
        s = N.QuartzPages()
        s.data, (s.stride_page, s.stride_slot, s.stride_head) = P, st
        sides.append(s)
    return N.QuartzPagedCache(N.PAGES_F16, page, heads, 128, pages, *sides)


ZERO = [(0, 256, 128), (4096, 0, 128), (4096, 256, 0)]


@pytest.mark.parametrize("strides", ZERO)
@pytest.mark.parametrize("side", ["k", "v"])
def test_written_pages(lib, strides, side):
    c = _cache(**{side: strides})
    assert lib.quartz_paged_append(C.byref(c), P, 256, 128, P, 256, 128, 1, P, None, None) == BAD
    assert lib.quartz_cache_compact(C.byref(c), 1, P, 4, None, 0, P, 64, P, 8, None, 0, 0, None) == BAD
    # attention only reads them: taken, up to the workspace
    assert lib.quartz_paged_attention(P, 256, 128, 1, 2, C.byref(c), P, 4, P, 64, 0, 1.0, P, 0, None, 0, 0, P, 0, None) == WS


@pytest.mark.parametrize("strides", [(0, 128), (256, 0)])
def test_rotated(lib, strides):
    r = N.QuartzRope(P, P, 64, 0, 0, 1.0)
    assert lib.quartz_rope(P, 256, 128, P, *strides, 0, 3, 2, 128, C.byref(r), None) == BAD


@pytest.mark.parametrize("strides", [(0, 64), (128, 0)])
def test_weights(lib, strides):
    c = _cache()
    assert lib.quartz_paged_attention(P, 256, 128, 2, 2, C.byref(c), P, 4, P, 64, 0, 1.0, P, 0, P, *strides, P, 1 << 30,
                                      None) == BAD
    assert lib.quartz_cache_compact(C.byref(c), 2, P, 4, None, 0, P, 64, P, 8, P, *strides, None) == BAD


@pytest.mark.gpu
def test_of_one_and_of_what_is_read():
    """A stride of a dimension of one is any number; repeated pages may be read."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    freqs, pos = Q.rope_frequencies(64)[0], torch.zeros(1, dtype=torch.int64, device="cuda")
    x = torch.randn(1, 1, 64, device="cuda")
    out = torch.empty(64, device="cuda").as_strided((1, 1, 64), (0, 0, 1))
    assert torch.equal(Q.rope(x, pos, freqs, out=out), x)
    with pytest.raises(Q.QuartzError):
        Q.rope(x.expand(2, 1, 64), pos.expand(2).contiguous(), freqs, out=out.expand(2, 1, 64))
    row = torch.randn(1, 1, 1, 64, device="cuda").half()
    c = Q.PagedCache(row.expand(3, 16, 2, 64), row.expand(3, 16, 2, 64), 16)
    table, lens = torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([40], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 2, 64, device="cuda").half()
    # the mean of equal rows: three parts of the type's half step
    o = Q.attention_paged(q, c, table, lens, 0.1)
    assert bool(((o - row[0, 0]).abs() <= row[0, 0].abs() * 2.0 ** -10).all()) and Q.device_status() == 0
    k = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(Q.QuartzError):
        Q.paged_append(c, k, k, torch.zeros(1, dtype=torch.int64, device="cuda"))
