"""Calls that the paged cache's documentation allows and that are far from the
ordinary: captured evictions, broadcast inputs, sides of different layouts, the
most sequences and heads."""
import pytest

import paged_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _planes(c):
    if hasattr(c.k, "codes"):
        return [t for e in (c.k, c.v) for t in (e.codes, e.flags, e.scales)]
    return [c.k, c.v]


@pytest.mark.parametrize("store", ["bf16", "lzs"])
@pytest.mark.parametrize("moved", [False, True])
def test_a_captured_eviction(Q, store, moved):
    """The choice and the closing-up in one graph, replayed over other weights and lengths: as the eager calls."""
    B, H, D, page, width, budget = 3, 2, 64, 16, 6, 40
    kw = dict(params=Q.Params(group_s=16)) if store == "lzs" else dict(dtype=torch.bfloat16)
    caches = [Q.empty_paged_cache(2 * B * width, page, H, D, **kw) for _ in range(2)]
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width)
    new_table = table + B * width if moved else None
    w, ln = torch.zeros(B, H, width * page, device="cuda"), torch.full((B,), 50, dtype=torch.int32, device="cuda")
    held = caches[1]

    def step():
        kept, new = Q.evict_select(w, ln, budget, recent=5, sinks=2)
        Q.cache_compact(held, table, ln, kept, new, new_table=new_table, weights=w)
        return kept, new

    for t in _planes(held):
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept, new = step()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for lens in ([96, 0, 41], [40, 77, 96], [1, 2, 39]):
        weights = torch.rand(B, H, width * page, generator=gen, device="cuda")
        lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        for a, b in zip(*map(_planes, caches)):
            a.view(torch.uint8).copy_(torch.randint(0, 256, a.view(torch.uint8).shape, generator=gen, device="cuda", dtype=torch.uint8))
            b.copy_(a)
        eager_w = weights.clone()
        want_kept, want_new = Q.evict_select(eager_w, lengths, budget, recent=5, sinks=2)
        Q.cache_compact(caches[0], table, lengths, want_kept, want_new, new_table=new_table, weights=eager_w)
        w.copy_(weights)
        ln.copy_(lengths)
        g.replay()
        assert torch.equal(kept, want_kept) and torch.equal(new, want_new) and torch.equal(w, eager_w)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*map(_planes, caches)))
    assert Q.device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_broadcast_inputs(Q, dtype):
    """Expanded tensors: one head's rows for all heads, one token's for all tokens."""
    T, H, D = 9, 5, 64
    freqs, pos = Q.rope_frequencies(48)[0], torch.arange(T, device="cuda") * 1000
    base = torch.randn(T, 1, D, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    heads = base.expand(T, H, D)
    assert torch.equal(Q.rope(heads, pos, freqs), Q.rope(heads.contiguous(), pos, freqs))
    token = base[:1].expand(T, H, D)
    assert torch.equal(Q.rope(token, pos, freqs, backward=True), Q.rope(token.contiguous(), pos, freqs, backward=True))
    if dtype != torch.float16:
        return
    slots, table = torch.arange(T, device="cuda"), torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    lens = torch.arange(1, T + 1, dtype=torch.int32, device="cuda")
    caches = []
    for k, v in ((heads, token), (heads.contiguous(), token.contiguous())):
        c = Q.empty_paged_cache(1, 16, H, D, dtype=dtype)
        Q.paged_append(c, k, v, slots, positions=pos, freqs=freqs)
        caches.append(c)
    a, b = caches
    assert torch.equal(a.k[0, :T], b.k[0, :T]) and torch.equal(a.v[0, :T], b.v[0, :T])
    # one row of the table and one query for all sequences
    one = table[:1].expand(T, 1)
    assert torch.equal(Q.attention_paged(token, a, one, lens, 0.1), Q.attention_paged(token.contiguous(), a, table, lens, 0.1))
    assert Q.device_status() == 0


def test_sides_of_different_layouts(Q):
    """Keys by slots, values by heads and in a wider pool: strides are each side's own."""
    pages, page, H, D, lens = 12, 8, 3, 128, [60, 17]
    k = torch.zeros(pages, page, H, D, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(pages, H + 2, page, D + 8, dtype=torch.bfloat16, device="cuda")
    c = Q.PagedCache(k, wide[:, 1:1 + H, :, :D].transpose(1, 2), page)
    plain = Q.empty_paged_cache(pages, page, H, D, dtype=torch.bfloat16)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(3), dtype=torch.int64)[:12].int().view(2, 6)
    table = torch.cat([table, table.flip(0)[:, :2]], 1).cuda()  # the second's last places are not used
    lens = [min(n, 48) for n in lens]
    slots = torch.cat([table.cpu().long()[b][torch.arange(n) // page] * page + torch.arange(n) % page for b, n in enumerate(lens)]).cuda()
    g = torch.Generator().manual_seed(4)
    x, y = (torch.randn(sum(lens), H, D, generator=g).bfloat16().cuda() for _ in range(2))
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = torch.randn(2, 2 * H, D, generator=g).bfloat16().cuda()
    w = torch.rand(2, H, 64, generator=g).cuda()
    for cache in (c, plain):
        Q.paged_append(cache, x, y, slots)
    kept, new = Q.evict_select(w, ln, 20, recent=3, sinks=1)
    for table_, lengths in ((table, ln), (table, new)):
        a, b = (Q.attention_paged(q, cache, table_, lengths, 0.1, max_len=48) for cache in (c, plain))
        assert torch.equal(a, b) and bool(a.isfinite().all())
        for cache in (c, plain):
            Q.cache_compact(cache, table, ln, kept, max_len=48)
    assert Q.device_status() == 0 and not wide[:, 0].any() and not wide[:, 4].any() and not wide[..., D:].any()


@pytest.mark.parametrize("store", ["f16", "lzs"])
def test_the_most_sequences(Q, store):
    """65535 sequences of 0, 1 or 2 tokens."""
    B, D, page = 65535, 64, 2
    kw = dict(params=Q.Params(group_s=16)) if store == "lzs" else dict(dtype=torch.float16)
    c = Q.empty_paged_cache(B, page, 1, D, **kw)
    g = torch.Generator(device="cuda").manual_seed(5)
    lens = torch.randint(0, 3, (B,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.randperm(B, generator=g, device="cuda", dtype=torch.int32)[:, None]
    x = torch.randn(B * 2, 1, D, generator=g, device="cuda").half()
    slots = (table.long() * 2 + torch.arange(2, device="cuda")).view(-1)
    Q.paged_append(c, x, x, slots)
    w = torch.zeros(B, 1, 2, device="cuda")
    q = torch.zeros(B, 1, D, dtype=torch.float16, device="cuda")  # every token weighs the same
    o = Q.attention_paged(q, c, table, lens, 1.0, out_dtype=torch.float32, weights=w)
    held = R.held(c)[1][table[:, 0].cpu().long(), :, 0]
    n = lens.cpu().double()[:, None]
    seen = torch.arange(2) < n
    want = (held * seen[..., None]).sum(1) / n.clamp(min=1)
    # halves and ones are exact; a sum of two and the division: 2 * 2^-24, and the exponential's 2^-22
    assert bool(((o[:, 0].cpu().double() - want).abs() <= (held.abs() * seen[..., None]).sum(1) * 2.0 ** -20).all())
    assert bool(((w[:, 0].cpu().double() - seen / n.clamp(min=1)).abs() <= 2.0 ** -20).all())
    # of two tokens the heavier stays (ties: the first)
    w = torch.randint(0, 2, (B, 1, 2), generator=g, device="cuda").float()
    before = [t.clone() for t in _planes(c)]
    kept, new = Q.evict_select(w, lens, 1)
    second = (lens == 2) & (w[:, 0, 1] > w[:, 0, 0])
    assert torch.equal(kept[:, 0, 0], torch.where(lens == 0, -1, second.int())) and torch.equal(new, lens.clamp(max=1))
    Q.cache_compact(c, table, lens, kept)
    rows = table[:, 0].long() * 2
    for a, b in zip(_planes(c), before):
        a, b = (t.view(2 * B, -1).view(torch.uint8) for t in (a, b))
        assert torch.equal(a[rows], b[rows + second]) and torch.equal(a[rows + 1], b[rows + 1])
    assert Q.device_status() == 0


def test_the_most_heads(Q):
    """1024 key heads; 65535 heads of a rotation."""
    H, D, n = 1024, 64, 5
    c = Q.empty_paged_cache(n, 1, H, D, dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(n, H, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.tensor([[3, 1, 4, 0, 2]], dtype=torch.int32, device="cuda")
    freqs, pos = Q.rope_frequencies(D)[0], torch.arange(n, device="cuda")
    Q.paged_append(c, k, v, table[0].long(), positions=pos, freqs=freqs)
    q = torch.randn(1, 2 * H, D, generator=g, device="cuda").bfloat16()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    o = Q.attention_paged(q, c, table, lens, 0.125, out_dtype=torch.float32)
    kh, vh = R.held(c)
    ref, add, mag, pv = R.attention(q.cpu(), kh, vh, table.cpu(), lens.cpu(), 0.125)
    bound, _ = R.attention_bounds(mag, pv, ref, add, n, D, 2, torch.float32, 17, float(vh.abs().max()))
    assert bool(((o.cpu().double() - ref).abs() <= bound).all())
    w = torch.rand(1, H, n, generator=g, device="cuda")
    kept, _ = Q.evict_select(w, lens, 3, recent=1)
    assert torch.equal(kept.cpu(), R.evict(w, lens, 3, 1, 0)[0])
    Q.cache_compact(c, table, lens, kept)
    rows, heads = table[0].long(), torch.arange(H, device="cuda")
    turned = Q.rope(k, pos, freqs)
    for j in range(3):
        src = kept[0, :, j].long()
        assert torch.equal(c.k[rows[j], 0], turned[src, heads]) and torch.equal(c.v[rows[j], 0], v[src, heads])
    x = torch.randn(2, 65535, 8, generator=g, device="cuda")
    y = Q.rope(x, pos[:2], freqs[:4])
    assert torch.equal(y[:, ::13107], Q.rope(x[:, ::13107].contiguous(), pos[:2], freqs[:4])) and Q.device_status() == 0
