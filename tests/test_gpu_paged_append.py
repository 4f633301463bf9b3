"""The append into pages: the encoder's and the rotation's bits in the right
places, and nothing anywhere else."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _new(T, H, D, dtype, seed, fused=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, (H + 3) if fused else H, D, generator=g)
    x[..., 5] *= 20
    return x.to(dtype).cuda()[:, :H] if fused else x.to(dtype).cuda()


def _slots(T, total, seed, skip=()):
    g = torch.Generator().manual_seed(seed)
    s = torch.randperm(total, generator=g)[:T]
    for i in skip:
        s[i] = -1
    return s


def _filled(Q, pages, page, H, D, dtype=None, params=None, heads_first=False):
    """A cache full of a pattern, and copies of it."""
    if params is not None:
        c = Q.empty_paged_cache(pages, page, H, D, params=params)
        ts = [t for e in (c.k, c.v) for t in (e.codes, e.flags, e.scales)]
    else:
        if heads_first:
            k, v = (torch.empty(pages, H, page, D, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2))
            c = Q.PagedCache(k, v, page)
        else:
            c = Q.empty_paged_cache(pages, page, H, D, dtype=dtype)
        ts = [c.k, c.v]
    for i, t in enumerate(ts):
        t.fill_(i + 1)
    return c, ts


@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("T,H,D,page,heads_first,fused", [(1, 1, 64, 1, False, False), (5, 3, 128, 16, False, True),
                                                          (37, 2, 192, 8, True, False), (9, 20, 256, 4, True, True)])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (-1, False), (-1, True), (40, False), (36, True)])
def test_16bit_pages(Q, dt, T, H, D, page, heads_first, fused, rotary, interleaved):
    dtype, pages = DTYPES[dt], (T + 5 + page - 1) // page + 1
    c, (kt, vt) = _filled(Q, pages, page, H, D, dtype, heads_first=heads_first)
    k, v = _new(T, H, D, dtype, 1, fused), _new(T, H, D, dtype, 2, fused)
    slots = _slots(T, pages * page, 3, skip=(1,) if T > 1 else ())
    want_k, want_v = kt.clone(), vt.clone()
    kk = k
    args = {}
    if rotary:
        freqs = Q.rope_frequencies(D if rotary < 0 else rotary)[0]
        pos = (torch.arange(T) * 977 + 60000).cuda()
        kk = Q.rope(k, pos, freqs, interleaved=interleaved, scale=1.1)
        args = dict(positions=pos, freqs=freqs, interleaved=interleaved, rope_scale=1.1)
    for t in range(T):
        s = int(slots[t])
        if s >= 0:
            want_k[s // page, s % page], want_v[s // page, s % page] = kk[t], v[t]
    Q.paged_append(c, k, v, slots.cuda(), **args)
    assert Q.device_status() == 0
    assert torch.equal(kt, want_k) and torch.equal(vt, want_v)


@pytest.mark.parametrize("gs", [8, 16, 32, 64])
@pytest.mark.parametrize("T,H,D,page,rope", [(1, 1, 64, 16, False), (6, 5, 128, 8, True), (33, 2, 192, 1, False),
                                             (11, 17, 256, 32, True)])
def test_encoded_pages(Q, gs, T, H, D, page, rope):
    pages = (T + 3 + page - 1) // page + 1
    c, ts = _filled(Q, pages, page, H, D, params=Q.Params(group_s=gs))
    k, v = _new(T, H, D, torch.float16, 4, True), _new(T, H, D, torch.float16, 5)
    v[0] = 0                                              # groups whose scale is 0
    slots = _slots(T, pages * page, 6, skip=(2,) if T > 2 else ())
    args = {}
    kk = k
    if rope:
        freqs, pos = Q.rope_frequencies(D // 2)[0], (torch.arange(T) * 31 + 5).cuda()
        kk = Q.rope(k, pos, freqs)
        args = dict(positions=pos, freqs=freqs)
    want = [t.clone() for t in ts]
    for i, x in enumerate((kk, v)):
        e = Q.quantize(x.contiguous().view(T * H, D), group_s=gs)
        for t in range(T):
            s = int(slots[t])
            if s < 0:
                continue
            rows = (s // page * H + torch.arange(H)) * page + s % page
            for dst, src in zip(want[3 * i:3 * i + 3], (e.codes, e.flags, e.scales)):
                dst[rows.cuda()] = src[t * H:(t + 1) * H]
    Q.paged_append(c, k, v, slots.cuda(), **args)
    assert Q.device_status() == 0
    for got, exp in zip(ts, want):
        assert torch.equal(got, exp)


@pytest.mark.parametrize("store", ["f16", "bf16", 8, 16, 32, 64])
@pytest.mark.parametrize("H,D", [(17, 64), (16, 128), (3, 128), (5, 192), (7, 256)])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (-1, False), (-1, True), (48, False)])
def test_many_tokens(Q, store, H, D, rotary, interleaved, T=None):
    """Enough tokens for every SM, where a thread takes units that are each other's partners and several tokens share a
    CTA; an odd number of tokens, some without a slot, keys inside a fused projection: the bits of rope() and quantize()."""
    T, page = T or 152 * 1024 * 32 // (H * D) + 13, 16
    total = (T + 40) // page + 1
    dtype = DTYPES.get(store, torch.float16)
    encoded = not isinstance(store, str)
    c, ts = _filled(Q, total, page, H, D, dtype, Q.Params(group_s=store) if encoded else None, heads_first=D == 192)
    k, v = _new(T, H, D, dtype, 21, True), _new(T, H, D, dtype, 22)
    slots = _slots(T, total * page, 23, skip=(0, 7, T - 1))
    want, kk, args = [t.clone() for t in ts], k, {}
    if rotary:
        freqs, pos = Q.rope_frequencies(D if rotary < 0 else rotary)[0], (torch.arange(T) * 3 + 9).cuda()
        kk = Q.rope(k, pos, freqs, interleaved=interleaved, scale=0.9)
        args = dict(positions=pos, freqs=freqs, interleaved=interleaved, rope_scale=0.9)
    there = slots >= 0
    at = slots[there]
    for i, x in enumerate((kk, v)):
        x = x[there.cuda()]
        if encoded:
            e = Q.quantize(x.reshape(-1, D), group_s=store)
            rows = ((at // page * H)[:, None] + torch.arange(H)).mul(page).add((at % page)[:, None]).view(-1).cuda()
            for dst, src in zip(want[3 * i:3 * i + 3], (e.codes, e.flags, e.scales)):
                dst[rows] = src
        else:
            want[i][(at // page).cuda(), (at % page).cuda()] = x
    Q.paged_append(c, k, v, slots.cuda(), **args)
    assert Q.device_status() == 0
    for got, exp in zip(ts, want):
        assert torch.equal(got, exp)


@pytest.mark.parametrize("store", ["bf16", 16])
@pytest.mark.parametrize("T,H,D", [(303, 8, 128), (305, 8, 128), (1217, 2, 128), (2433, 1, 256), (4871, 1, 64), (1300, 3, 192)])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (-1, False), (-1, True), (16, False), (20, False)])
def test_some_tokens(Q, store, T, H, D, rotary, interleaved):
    """Both sides of the sizes from which on a CTA takes keys and values, and several tokens."""
    test_many_tokens(Q, store, H, D, rotary, interleaved, T)


def test_slot_out_of_range_is_reported_and_not_followed(Q):
    c, ts = _filled(Q, 2, 8, 2, 64, torch.float16)
    before = [t.clone() for t in ts]
    k = _new(3, 2, 64, torch.float16, 7)
    for bad in (16, 1 << 40, 2 ** 62):
        Q.paged_append(c, k, k, torch.tensor([bad, -1, -(1 << 50)], device="cuda"))
        assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX and Q.device_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(ts, before))


def test_empty_and_refusals(Q):
    c, _ = _filled(Q, 2, 8, 2, 64, torch.float16)
    k = _new(3, 2, 64, torch.float16, 8)
    slots = torch.arange(3, device="cuda")
    Q.paged_append(c, k[:0], k[:0], slots[:0])
    pos, freqs = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.ones(16, dtype=torch.float64, device="cuda")
    for bad in (lambda: Q.paged_append(c, k.bfloat16(), k, slots), lambda: Q.paged_append(c, k, k[:2], slots),
                lambda: Q.paged_append(c, k, k, slots.int()), lambda: Q.paged_append(c, k, k, slots, positions=pos),
                lambda: Q.paged_append(c, k, k, slots, freqs=freqs), lambda: Q.paged_append(c, k[:, :1], k[:, :1], slots)):
        with pytest.raises(ValueError):
            bad()
    odd = torch.empty(3 * 2 * 64 + 1, dtype=torch.float16, device="cuda")[1:].view(3, 2, 64)
    with pytest.raises(Q.QuartzError):
        Q.paged_append(c, odd, k, slots)
    with pytest.raises(ValueError):
        Q.PagedCache(c.k, c.v, 12)
    with pytest.raises(ValueError):
        Q.PagedCache(c.k, c.v.bfloat16(), 8)
    e = Q.empty_encoded(2 * 8 * 2, 64)
    with pytest.raises(ValueError):
        Q.PagedCache(e, e, 8)                             # heads are needed
