"""Eviction: the choice against a sort, the closing-up against indexing; both exact."""
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


def _weights(B, H, n, seed, kind="sums"):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(1.5 * torch.randn(B, H, n, generator=g))
    if kind == "ties":
        w = torch.randint(0, 3, (B, H, n), generator=g).float()
    elif kind == "odd":
        special = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 1.0, -1.0, 3e38])
        w = special[torch.randint(0, len(special), (B, H, n), generator=g)]
    elif kind == "equal":
        w = torch.full((B, H, n), 0.25)
    return w


# (lens, budget, recent, sinks): nothing to do, one too many, only the fixed ones, none fixed, budget one
CASES = [([0, 1, 7, 8, 9, 40], 8, 2, 1), ([100, 33, 64], 32, 32, 0), ([100, 33, 64], 32, 0, 32), ([100, 33], 32, 28, 4),
         ([500, 1, 31], 1, 0, 0), ([1000, 999, 3], 600, 0, 0), ([4097, 2048], 2047, 100, 4), ([50], 100, 10, 2)]


@pytest.mark.parametrize("lens,budget,recent,sinks", CASES)
@pytest.mark.parametrize("kind", ["sums", "ties", "odd", "equal"])
def test_select(Q, lens, budget, recent, sinks, kind):
    H, n = 3, max(lens) + 5
    w, ln = _weights(len(lens), H, n, 1, kind), torch.tensor(lens, dtype=torch.int32)
    kept, new = Q.evict_select(w.cuda(), ln.cuda(), budget, recent=recent, sinks=sinks)
    assert Q.device_status() == 0
    want, want_new = R.evict(w, ln, budget, recent, sinks)
    assert torch.equal(kept.cpu(), want) and torch.equal(new.cpu(), want_new)


@pytest.mark.parametrize("n", [20000, 48 * 1024, 48 * 1024 + 1, 70001])
def test_select_long(Q, n):
    """Around what a CTA holds in shared memory, with strided weights and a stated bound."""
    w = _weights(2, 4, n + 7, 2)
    ln = torch.tensor([n, n - 1234], dtype=torch.int32)
    view = w.cuda()[:, 1:3]
    kept, _ = Q.evict_select(view, ln.cuda(), n // 3, recent=100, sinks=4, max_len=n)
    want, _ = R.evict(w[:, 1:3], ln, n // 3, 100, 4)
    assert torch.equal(kept.cpu(), want)


def test_select_bad_length_is_reported(Q):
    w = _weights(2, 2, 64, 3).cuda()
    for bad in (65, -3):
        Q.evict_select(w, torch.tensor([bad, 20], dtype=torch.int32, device="cuda"), 8)
        assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX


def test_select_refusals(Q):
    w, ln = _weights(2, 2, 64, 4).cuda(), torch.tensor([60, 20], dtype=torch.int32, device="cuda")
    for bad in (lambda: Q.evict_select(w.double(), ln, 8), lambda: Q.evict_select(w, ln[:1], 8),
                lambda: Q.evict_select(w, ln.long(), 8), lambda: Q.evict_select(w, ln, 8, max_len=65),
                lambda: Q.evict_select(w, ln, 8, kept=torch.empty(2, 2, 9, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: Q.evict_select(w, ln, 8, recent=9), lambda: Q.evict_select(w, ln, 8, recent=-1),
                lambda: Q.evict_select(w, ln, 8, recent=5, sinks=4)):
        with pytest.raises(Q.QuartzError):
            bad()


def _cache(Q, store, pages, page, H, D, gs=16):
    g = torch.Generator(device="cuda").manual_seed(5)
    if store == "lzs":
        c = Q.empty_paged_cache(pages, page, H, D, params=Q.Params(group_s=gs))
        ts = [t for e in (c.k, c.v) for t in (e.codes, e.flags, e.scales)]
        for t in ts:
            t.view(torch.uint8).copy_(torch.randint(0, 256, t.view(torch.uint8).shape, generator=g, device="cuda",
                                                    dtype=torch.uint8))
        views = [t.view(pages, H, page, -1).transpose(1, 2) for t in ts]
    else:
        dtype = {"f16": torch.float16, "bf16": torch.bfloat16}[store]
        shape = (pages, H, page, D) if page % 8 else (pages, page, H, D)
        k, v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
        if page % 8:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        c = Q.PagedCache(k, v, page)
        views = [k, v]
    return c, views


def _bits(views):
    return [v.contiguous().view(torch.uint8).clone() for v in views]


@pytest.mark.parametrize("store,H,D,page,gs", [("f16", 2, 64, 16, 16), ("bf16", 3, 192, 4, 16), ("f16", 1, 256, 1, 16),
                                               ("lzs", 2, 128, 16, 16), ("lzs", 3, 64, 8, 64), ("lzs", 1, 192, 32, 8),
                                               ("lzs", 2, 256, 2, 32)])
@pytest.mark.parametrize("moved", [False, True])
@pytest.mark.parametrize("lens,budget", [([0, 1, 20, 37], 20), ([700, 333], 300), ([2500], 2400)])
def test_compact(Q, store, H, D, page, gs, moved, lens, budget):
    need = [-(-n // page) for n in lens]
    fresh = [-(-min(n, budget) // page) for n in lens]
    total = sum(need) + sum(fresh) + 1
    c, views = _cache(Q, store, total, page, H, D, gs)
    g = torch.Generator().manual_seed(6)
    order = torch.randperm(total, generator=g, dtype=torch.int32)
    width = max(need + [1])
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    new_table = torch.full((len(lens), -(-budget // page)), -1, dtype=torch.int32)
    at = 0
    for b in range(len(lens)):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        new_table[b, :fresh[b]] = order[at:at + fresh[b]]
        at += fresh[b]
    w = _weights(len(lens), H, width * page + 2, 7)
    ln = torch.tensor(lens, dtype=torch.int32)
    kept, new = Q.evict_select(w.cuda(), ln.cuda(), budget, recent=3, sinks=1, max_len=width * page)
    before = _bits(views)
    want = [x.clone() for x in before]
    want_w = w.clone()
    to = new_table if moved else table
    kc = kept.cpu()
    for b, n in enumerate(lens):
        m = min(n, budget)
        for h in range(H):
            src, j = kc[b, h, :m].long(), torch.arange(m)
            for x, y in zip(before, want):
                y[to[b].long()[j // page], j % page, h] = x[table[b].long()[src // page], src % page, h].to(y.device)
            want_w[b, h, :m] = w[b, h, src]
            want_w[b, h, m:n] = 0
    wc = w.cuda()
    Q.cache_compact(c, table.cuda(), ln.cuda(), kept, new, new_table=new_table.cuda() if moved else None, weights=wc)
    assert Q.device_status() == 0
    for got, exp in zip(_bits(views), want):
        assert torch.equal(got, exp)
    assert torch.equal(wc.cpu(), want_w)


def test_compact_bad_indices_are_reported_and_not_followed(Q):
    c, views = _cache(Q, "f16", 8, 16, 2, 64)
    table = torch.arange(4, dtype=torch.int32)[None]
    ln = torch.tensor([60], dtype=torch.int32)
    kept, _ = Q.evict_select(_weights(1, 2, 64, 8).cuda(), ln.cuda(), 10)
    before = _bits(views)
    for where, value in ((0, 60), (1, -1), (2, 2 ** 31 - 1)):
        k = kept.clone()
        k[0, 0, where] = value
        Q.cache_compact(c, table.cuda(), ln.cuda(), k, new_table=torch.tensor([[4]], dtype=torch.int32, device="cuda"))
        assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX
    for t, nt in ((torch.tensor([[0, 1, 2, 8]]), [[4]]), (torch.tensor([[0, -1, 2, 3]]), [[4]]), (table, [[9]])):
        Q.cache_compact(c, t.int().cuda(), ln.cuda(), kept, new_table=torch.tensor(nt, dtype=torch.int32, device="cuda"))
    assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX
    after = _bits(views)
    keep = [0, 1, 2, 3, 5, 6, 7]                         # only page 4 was written
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(after, before))


def test_compact_refusals(Q):
    c, _ = _cache(Q, "f16", 8, 16, 2, 64)
    table, ln = torch.arange(4, dtype=torch.int32, device="cuda")[None], torch.tensor([60], dtype=torch.int32, device="cuda")
    w = _weights(1, 2, 64, 9).cuda()
    kept, _ = Q.evict_select(w, ln, 40)
    for bad in (lambda: Q.cache_compact(c, table, ln, kept[:, :1]), lambda: Q.cache_compact(c, table.long(), ln, kept),
                lambda: Q.cache_compact(c, table, ln, kept, new_table=table[:, :2]),
                lambda: Q.cache_compact(c, table, ln, kept, weights=w[..., :32]),
                lambda: Q.cache_compact(c, table, ln, kept, max_len=65)):
        with pytest.raises(ValueError):
            bad()
