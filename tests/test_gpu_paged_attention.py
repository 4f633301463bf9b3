"""Attention of one new token over pages against the definition in 64 bits."""
import pytest

import paged_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
OUT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def make_cache(Q, lens, H, D, page, store, gs=16, seed=0, heads_first=False, size=1.0, poison=True):
    """A pool whose pages hold the sequences' tokens in a shuffled order; what
    belongs to no token is infinite or NaN (16-bit pages)."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    total = sum(need) + 2
    order = torch.randperm(total, generator=g, dtype=torch.int32)
    width = max(need + [1]) + 1
    table = torch.full((len(lens), width), -7, dtype=torch.int32)
    slots, at = [], 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
        t = torch.arange(lens[b])
        slots.append(table[b].long()[t // page] * page + t % page)
    slots = torch.cat(slots) if slots else torch.zeros(0, dtype=torch.int64)
    dtype = {"f16": torch.float16, "bf16": torch.bfloat16, "lzs": torch.float16}[store]
    if store == "lzs":
        c = Q.empty_paged_cache(total, page, H, D, params=Q.Params(group_s=gs))
        for e in (c.k, c.v):
            e.codes.fill_(0x77)
            e.flags.fill_(4)
            e.scales.fill_(float("inf") if poison else 0.0)
    elif heads_first:
        k, v = (torch.empty(total, H, page, D, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2))
        c = Q.PagedCache(k, v, page)
    else:
        c = Q.empty_paged_cache(total, page, H, D, dtype=dtype)
    if store != "lzs":
        c.k.fill_(float("nan") if poison else 0.0)
        c.v.fill_(float("inf") if poison else 0.0)
    k, v = (torch.randn(len(slots), H, D, generator=g) * size for _ in range(2))
    k[..., 3] *= 6
    Q.paged_append(c, k.to(dtype).cuda(), v.to(dtype).cuda(), slots.cuda())
    return c, table, torch.tensor(lens, dtype=torch.int32)


def _q(B, Hq, D, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(B, Hq, D, generator=g) * size).to(dtype)


def check(Q, c, table, lens, q, scale, window=0, out="f32", weights=False, store="f16", max_len=None, group=1):
    width = table.shape[1] * c.page_size
    w = w0 = None
    if weights:
        w0 = torch.rand(len(lens), c.heads, width + 3, generator=torch.Generator().manual_seed(5))
        w = w0.cuda()
    o = Q.attention_paged(q.cuda(), c, table.cuda(), lens.cuda(), scale, window=window, out_dtype=OUT[out], weights=w,
                          max_len=max_len)
    assert Q.device_status() == 0
    k, v = R.held(c)
    ref, add, mag, pv = R.attention(q, k, v, table, lens, scale, window)
    bits = 22 if store == "f16" else 17
    bound, w_rel = R.attention_bounds(mag, pv, ref, add, int(lens.max()) if len(lens) else 0, c.dim, q.shape[1] // c.heads,
                                      OUT[out], bits, float(v.nan_to_num(0, 0, 0).abs().max()))
    assert o.dtype == OUT[out]
    err = (o.cpu().double() - ref).abs()
    assert bool((err <= bound).all()), float((err - bound).max())
    if weights:
        got = w.cpu().double()
        want = w0.double()
        want[..., :width] += add
        # the bound on the addition, and half a step of the sum
        tol = torch.zeros_like(want)
        tol[..., :width] = add * w_rel[..., None]
        tol += want.abs() * 2.0 ** -24 + group * 2.0 ** -126
        assert bool(((got - want).abs() <= tol).all())
        for b, n in enumerate(lens.tolist()):           # past the tokens, and before the window: as they were
            first = max(0, n - window) if window else 0
            assert torch.equal(w.cpu()[b, :, n:], w0[b, :, n:]) and torch.equal(w.cpu()[b, :, :first], w0[b, :, :first])
    return o


# (lens, kv heads, group, dim, page): lengths 0 and 1, tile and page ends, one long; groups over 8; MHA and MQA
SHAPES = [([1], 1, 1, 64, 16), ([0, 1, 15, 16, 17], 2, 4, 128, 16), ([63, 64, 65, 129], 1, 8, 128, 8),
          ([257, 0, 300], 3, 1, 64, 32), ([100, 1, 511], 1, 16, 128, 1), ([77, 200], 2, 7, 192, 4),
          ([33, 513], 1, 12, 256, 64), ([0, 0], 2, 2, 128, 16), ([1025], 4, 3, 256, 128), ([2500, 3], 1, 5, 64, 4096)]


@pytest.mark.parametrize("lens,H,group,D,page", SHAPES)
@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
@pytest.mark.parametrize("out,weights", [("f32", True), ("f16", False)])
def test_shapes(Q, lens, H, group, D, page, store, out, weights):
    c, table, ln = make_cache(Q, lens, H, D, page, store, seed=len(lens) + D, heads_first=page == 8)
    q = _q(len(lens), H * group, D, c.dtype, 3)
    check(Q, c, table, ln, q, D ** -0.5, out=out, weights=weights, store=store)


@pytest.mark.parametrize("gs", [8, 16, 32, 64])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_every_subgroup_and_width(Q, gs, D):
    c, table, ln = make_cache(Q, [150, 41], 2, D, 16, "lzs", gs, seed=gs + D)
    check(Q, c, table, ln, _q(2, 6, D, torch.float16, 4), D ** -0.5, store="lzs", weights=True, out="bf16")


@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
@pytest.mark.parametrize("window", [1, 7, 16, 100, 333, 1000])
def test_window(Q, store, window):
    c, table, ln = make_cache(Q, [333, 0, 5, 64, 200], 2, 128, 16, store, seed=window)
    check(Q, c, table, ln, _q(5, 8, 128, c.dtype, 5), 0.09, window=window, store=store, weights=True)


@pytest.mark.parametrize("store", ["f16", "lzs"])
@pytest.mark.parametrize("page", [1, 4, 8, 16, 32])
def test_pages_before_the_window_may_be_gone(Q, store, page):
    """A page none of whose tokens is in the window is not looked up: its place in the table may be free."""
    lens, window = [333, 50, 201], 45
    c, table, ln = make_cache(Q, lens, 2, 64, page, store, seed=page)
    q = _q(3, 4, 64, torch.float16, 18).cuda()
    want = Q.attention_paged(q, c, table.cuda(), ln.cuda(), 0.1, window=window)
    gone = table.clone()
    for b, n in enumerate(lens):
        gone[b, :max(0, n - window) // page] = -7
    assert torch.equal(Q.attention_paged(q, c, gone.cuda(), ln.cuda(), 0.1, window=window), want)
    assert Q.device_status() == 0


@pytest.mark.parametrize("store", ["f16", "lzs"])
def test_many_splits(Q, store):
    """One sequence cut into as many splits as there are SMs for; a short one beside it leaves most of them empty."""
    c, table, ln = make_cache(Q, [9001, 70], 1, 128, 16, store, seed=9)
    check(Q, c, table, ln, _q(2, 4, 128, torch.float16, 6), 128 ** -0.5, store=store, weights=True, out="f16")


@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
def test_large_scores_and_small_values(Q, store):
    """Scores of hundreds of nats (one token takes all), a negative scale, and values far below one."""
    for size, scale in ((4.0, 1.0), (4.0, -1.0), (0.004, 20.0)):
        c, table, ln = make_cache(Q, [300, 40], 2, 128, 16, store, seed=11, size=size)
        check(Q, c, table, ln, _q(2, 4, 128, c.dtype, 7, size), scale, store=store)


@pytest.mark.parametrize("store,size,scale", [("f16", 60000.0, 1e22), ("bf16", 2.0 ** 58, 1.0), ("lzs", 60000.0, 1e22)])
@pytest.mark.parametrize("lens,H", [([5, 900, 0, 1], 2), ([777], 40), ([3000] * 2, 8)])
def test_scores_far_below_zero(Q, store, size, scale, lens, H):
    """Equal scores of -1e33 and below (finite in binary32: -2^122 with bf16; with factors of 2^62 they would be -2^130),
    which no maximum to start from may hide: every token weighs the same.  The
    weights are 2^0 over their number, exact until the division and its sum: the bound is that of the values alone."""
    c, table, ln = make_cache(Q, lens, H, 64, 16, store, seed=20)
    total = int(ln.sum())
    slots = torch.cat([table[b].long()[torch.arange(n) // 16] * 16 + torch.arange(n) % 16 for b, n in enumerate(lens)])
    g = torch.Generator().manual_seed(21)
    v = torch.randn(total, H, 64, generator=g).to(c.dtype)
    Q.paged_append(c, torch.full((total, H, 64), size, dtype=c.dtype, device="cuda"), v.cuda(), slots.cuda())
    q = torch.full((len(lens), H, 64), -size, dtype=c.dtype)
    w = torch.zeros(len(lens), H, table.shape[1] * 16, device="cuda")
    a = Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), scale, out_dtype=torch.float32)
    b = Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), scale, out_dtype=torch.float32, weights=w)
    held = R.held(c)[1]
    for i, n in enumerate(lens):
        t = torch.arange(n)
        at = held[table[i].long()[t // 16], t % 16]
        want, mag = (at.mean(0), at.abs().mean(0)) if n else (torch.zeros(H, 64), torch.zeros(H, 64))
        # the weights' parts 2^-17, and n / 16 + 64 steps of 2^-23 in each of two sums
        for o in (a, b):
            assert bool(((o[i].cpu().double() - want).abs() <= mag * (2.0 ** -17 + 2 * (n / 16 + 64) * 2.0 ** -23)).all())
        got = w[i, :, :n].cpu().double()
        assert bool(((got * n - 1).abs() <= (n / 16 + 72) * 2.0 ** -23).all()) and not w[i, :, n:].any()
    assert Q.device_status() == 0


def test_a_sink_does_not_drown_small_weights(Q):
    """One token 17 nats ahead of 8000 others that together weigh 3e-4: their values are not lost below fp16's
    smallest weights."""
    D, n = 64, 8000
    c = Q.empty_paged_cache(n // 16, 16, 1, D, dtype=torch.float16)
    k = torch.zeros(n, 1, D, dtype=torch.float16)
    k[0, 0, 0] = 17.0
    v = torch.full((n, 1, D), 1000.0, dtype=torch.float16)
    v[0] = 0
    Q.paged_append(c, k.cuda(), v.cuda(), torch.arange(n, device="cuda"))
    table = torch.arange(n // 16, dtype=torch.int32)[None]
    q = torch.zeros(1, 1, D, dtype=torch.float16)
    q[..., 0] = 1.0
    check(Q, c, table, torch.tensor([n], dtype=torch.int32), q, 1.0, store="f16")


def test_known_bound_and_given_buffers(Q):
    c, table, ln = make_cache(Q, [40, 33], 2, 128, 16, "f16", seed=13)
    q = _q(2, 4, 128, torch.float16, 8)
    a = check(Q, c, table, ln, q, 0.1, max_len=40, out="f16")
    n = Q.attention_paged_workspace_size(c, 2, 4, 40)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = torch.empty(2, 4, 128, dtype=torch.float16, device="cuda")
    b = Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), 0.1, max_len=40, out=out, workspace=ws)
    assert b is out and torch.equal(a, out)
    with pytest.raises(Q.QuartzError):
        Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), 0.1, max_len=40, workspace=ws[:16])


def test_query_strides_and_shared_pages(Q):
    """Queries inside a fused projection; two sequences that share their first pages."""
    c, table, ln = make_cache(Q, [64, 100], 2, 128, 16, "bf16", seed=14)
    table[0, :4] = table[1, :4]
    fused = _q(2, 8, 128, torch.bfloat16, 9)
    check(Q, c, table, ln, fused[:, 2:6], 0.1, store="bf16")
    a = Q.attention_paged(fused.cuda()[:, 2:6], c, table.cuda(), ln.cuda(), 0.1)
    b = Q.attention_paged(fused[:, 2:6].contiguous().cuda(), c, table.cuda(), ln.cuda(), 0.1)
    assert torch.equal(a, b)


@pytest.mark.parametrize("store", ["f16", "lzs"])
def test_a_table_without_places(Q, store):
    """Sequences that have no page at all: zeros, and the sums as they were."""
    c, _, _ = make_cache(Q, [20], 2, 64, 16, store, seed=18)
    q = _q(3, 4, 64, torch.float16, 14).cuda()
    table, lens = torch.empty(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    w = torch.rand(3, 2, 5, device="cuda")
    before = w.clone()
    o = Q.attention_paged(q, c, table, lens, 0.1, weights=w)
    assert Q.device_status() == 0 and not o.any() and torch.equal(w, before)
    none = Q.attention_paged(q[:0], c, table[:0], lens[:0], 0.1)
    assert none.shape == (0, 4, 64)


@pytest.mark.parametrize("groups", [9, 16, 33])
def test_many_query_heads_per_key_head(Q, groups):
    """More heads than a CTA takes, and than the sums of weights hold at a time (65 below)."""
    c, table, ln = make_cache(Q, [70, 300], 1, 64, 16, "bf16", seed=groups)
    check(Q, c, table, ln, _q(2, groups, 64, torch.bfloat16, 15), 0.125, store="bf16", weights=True)


def test_more_query_heads_than_the_sums_hold(Q):
    c, table, ln = make_cache(Q, [40], 1, 64, 16, "f16", seed=19)
    check(Q, c, table, ln, _q(1, 65, 64, torch.float16, 16), 0.125, store="f16", weights=True)


@pytest.mark.parametrize("store", ["f16", "lzs"])
@pytest.mark.parametrize("B,H,n", [(1, 40, 777), (1, 1, 500), (2, 8, 3000), (200, 4, 90), (3, 16, 1100)])
def test_every_plan(Q, store, B, H, n):
    """One split, clusters, many splits with a join, and more heads than the SMs hold: against each other by the
    definition, ragged lengths included."""
    lens = [max(0, n - 37 * i % (n + 1)) for i in range(B)]
    c, table, ln = make_cache(Q, lens, H, 128, 16, store, seed=B + H)
    check(Q, c, table, ln, _q(B, H, 128, torch.float16, 17), 128 ** -0.5, store=store, out="f16")


@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
@pytest.mark.parametrize("lens,H,group,D,window", [([2500, 0, 1, 700], 1, 5, 128, 0), ([0, 0, 3000], 2, 9, 64, 0),
                                                   ([64 * i % 1500 for i in range(32)], 1, 2, 128, 0), ([0] * 5, 1, 1, 64, 0),
                                                   ([5000, 3000, 90], 1, 4, 192, 1100), ([2049], 2, 3, 256, 0)])
def test_few_sequences_share_a_wave(Q, store, lens, H, group, D, window):
    """CTAs given out by the lengths: empty sequences among them, a window, more heads than a CTA takes; the table's
    bound and a far larger one (the lengths count, not the bound)."""
    c, table, ln = make_cache(Q, lens, H, D, 16, store, seed=len(lens) + D)
    q = _q(len(lens), H * group, D, c.dtype, 18)
    check(Q, c, table, ln, q, D ** -0.5, window=window, store=store, out="f16")
    check(Q, c, table, ln, q, D ** -0.5, window=window, store=store, weights=True)
    wide = torch.cat([table, torch.full((len(lens), 500), -3, dtype=torch.int32)], 1)
    check(Q, c, wide, ln, q, D ** -0.5, window=window, store=store, out="f16")


def test_far_pages(Q):
    """Element offsets past 2^31 (and byte offsets past 2^32): a pool of 4.3 GB a side whose last pages are used."""
    pages, page, H, D = 2 ** 15 + 4, 64, 8, 128
    k, v = (torch.empty(pages, page, H, D, dtype=torch.float16, device="cuda") for _ in range(2))
    c = Q.PagedCache(k, v, page)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32)
    t = torch.arange(150)
    slots = table[0].long()[t // page] * page + t % page
    new = _q(150, H, D, torch.float16, 10)
    Q.paged_append(c, new.cuda(), new.flip(0).cuda(), slots.cuda())
    q, ln = _q(1, H, D, torch.float16, 11), torch.tensor([150], dtype=torch.int32)
    o = Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), 0.1)
    small = Q.empty_paged_cache(3, page, H, D, dtype=torch.float16)
    Q.paged_append(small, new.cuda(), new.flip(0).cuda(), t.cuda())
    want = Q.attention_paged(q.cuda(), small, torch.arange(3, dtype=torch.int32, device="cuda")[None], ln.cuda(), 0.1)
    assert Q.device_status() == 0 and torch.equal(o, want)


@pytest.mark.parametrize("store", ["f16", "lzs"])
def test_bad_pages_and_lengths_are_reported(Q, store):
    """A page outside the pool and a length past the bound are not followed; other sequences are untouched by it."""
    c, table, ln = make_cache(Q, [50, 50, 50], 2, 128, 16, store, seed=15, poison=False)
    q = _q(3, 4, 128, torch.float16, 12).cuda()
    good = Q.attention_paged(q, c, table.cuda(), ln.cuda(), 0.1, max_len=64)
    for row, value in ((0, c.num_pages), (2, -1), (1, 2 ** 31 - 1)):
        t = table.clone()
        t[row, 1] = value
        o = Q.attention_paged(q, c, t.cuda(), ln.cuda(), 0.1, max_len=64)
        assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX and Q.device_status() == 0
        others = [i for i in range(3) if i != row]
        assert torch.equal(o[others], good[others])
    for value in (65, -1):
        n = ln.clone()
        n[1] = value
        o = Q.attention_paged(q, c, table.clamp(min=0).cuda(), n.cuda(), 0.1, max_len=64)
        assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX
        assert torch.equal(o[[0, 2]], good[[0, 2]])


def test_refusals(Q):
    c, table, ln = make_cache(Q, [20, 20], 2, 64, 16, "f16", seed=16)
    q, tb, n = _q(2, 4, 64, torch.float16, 13).cuda(), table.cuda(), ln.cuda()
    w = torch.zeros(2, 2, tb.shape[1] * 16, device="cuda")
    for bad in (lambda: Q.attention_paged(q.bfloat16(), c, tb, n, 1.0), lambda: Q.attention_paged(q[:, :3], c, tb, n, 1.0),
                lambda: Q.attention_paged(q[:1], c, tb, n, 1.0), lambda: Q.attention_paged(q, c, tb.long(), n, 1.0),
                lambda: Q.attention_paged(q, c, tb, n.long(), 1.0), lambda: Q.attention_paged(q, c, tb, n, 1.0, max_len=1000),
                lambda: Q.attention_paged(q, c, tb, n, 1.0, weights=w[..., :16]),
                lambda: Q.attention_paged(q, c, tb, n, 1.0, weights=w.half()),
                lambda: Q.attention_paged(q, c, tb, n, 1.0, out=torch.empty(2, 4, 32, device="cuda")),
                lambda: Q.attention_paged(q, c, tb.cpu(), n, 1.0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: Q.attention_paged(q, c, tb, n, float("nan")), lambda: Q.attention_paged(q, c, tb, n, 1.0, window=-1)):
        with pytest.raises(Q.QuartzError):
            bad()
