"""The operators for several new tokens as a server uses them together: heads
normed and rotated, appended, prompts in chunks, drafted trees verified, decoding
one by one, eviction; and calls that no formula needs but a user makes."""
import pytest

from test_gpu_tokens_attention import Case, _trees

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

H, G, D, PAGE = 2, 4, 128, 16


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


class Server:
    def __init__(self, Q, store):
        self.Q = Q
        kw = dict(params=Q.Params(group_s=16)) if store == "lzs" else dict(dtype=torch.bfloat16)
        self.cache = Q.empty_paged_cache(40, PAGE, H, D, **kw)
        self.table = torch.randperm(40, generator=torch.Generator().manual_seed(1))[:36].view(2, 18).int().cuda()
        self.freqs, self.scale = Q.rope_frequencies(D, base=500000.0, scaling="yarn", factor=4.0, original_length=4096)
        g = torch.Generator().manual_seed(2)
        self.wq, self.wk = ((1 + 0.1 * torch.randn(D, generator=g)).cuda() for _ in range(2))
        self.lens = [0, 0]

    def new(self, ms, seed):
        """Queries, keys and values of ms[b] new tokens of each sequence, as a projection leaves them."""
        x = torch.randn(sum(ms), H * G + 2 * H, D, generator=torch.Generator().manual_seed(seed)).to(self.cache.dtype).cuda()
        return x[:, :H * G], x[:, H * G:-H], x[:, -H:]

    def add(self, ms, qkv, positions=None):
        """The new tokens normed, rotated and appended; their queries."""
        Q = self.Q
        at = torch.cat([torch.arange(n, n + m) for n, m in zip(self.lens, ms)]).cuda()
        which = torch.cat([torch.full((m,), b) for b, m in enumerate(ms)]).cuda()
        q, k = Q.qk_norm_rope(qkv[0], qkv[1], self.wq, self.wk, at if positions is None else positions, self.freqs, scale=self.scale)
        slots = self.table.long()[which, at // PAGE] * PAGE + at % PAGE
        Q.paged_append(self.cache, k, qkv[2], slots)
        self.lens = [n + m for n, m in zip(self.lens, ms)]
        return q

    def attend(self, q, ms, **how):
        starts = torch.tensor([0, ms[0], ms[0] + ms[1]], dtype=torch.int32).cuda()
        return self.Q.attention_paged_tokens(q, self.cache, self.table, torch.tensor(self.lens, dtype=torch.int32).cuda(), starts,
                                             D ** -0.5, out_dtype=torch.float32, **how)


@pytest.mark.parametrize("store", ["bf16", "lzs"])
def test_chunks_drafts_and_single_tokens_agree(Q, store):
    """A prompt in one call, in chunks, token by token and as a chain of drafted tokens: each is within the weights'
    rounding of the others (the bound of the definition, checked elsewhere, is that of two results apart: a half step of the
    type for every weight, and what binary32 sums of 128 and 200 terms add)."""
    ms = [150, 90]
    whole = Server(Q, store)
    qkv = whole.new(ms, 3)
    want = whole.attend(whole.add(ms, qkv), ms)
    tol = 2 * torch.finfo(whole.cache.dtype).eps * float(qkv[2].abs().max()) + 1e-4
    parts = Server(Q, store)
    done = [0, 0]
    for step in ([100, 1], [0, 40], [49, 48], [1, 1]):
        rows = torch.cat([torch.arange(o + d, o + d + m) for o, d, m in zip((0, ms[0]), done, step)]).cuda()
        piece = tuple(t[rows] for t in qkv)
        chain = [(1 << j + 1) - 1 for m in step for j in range(m)]
        q = parts.add(step, piece)
        got = [parts.attend(q, step)]
        if max(step) <= 64:
            tree = torch.tensor([c - (1 << 64) if c >> 63 else c for c in chain]).cuda()
            got.append(parts.attend(q, step, tree=tree))
        if step == [1, 1]:
            got.append(Q.attention_paged(q, parts.cache, parts.table, torch.tensor(parts.lens, dtype=torch.int32).cuda(), D ** -0.5,
                                         out_dtype=torch.float32))
        for o in got:
            assert float((o - want[rows]).abs().max()) <= tol
        done = [d + m for d, m in zip(done, step)]
    assert Q.device_status() == 0


@pytest.mark.parametrize("store", ["bf16", "lzs"])
def test_drafts_accepted_and_evicted(Q, store):
    """Siblings at one position do not see each other: a branch gives what it gives alone.  Then the accepted token is decoded
    and the cache evicted, with the sums of attention_paged."""
    s = Server(Q, store)
    s.attend(s.add([100, 60], s.new([100, 60], 1)), [100, 60])
    ms, qkv = [3, 3], s.new([3, 3], 2)
    positions = torch.tensor([100, 101, 101, 60, 61, 61]).cuda()  # a root and two children
    q = s.add(ms, qkv, positions)
    o = s.attend(q, ms, tree=torch.tensor([1, 3, 5] * 2).cuda())
    alone = Server(Q, store)
    alone.attend(alone.add([100, 60], alone.new([100, 60], 1)), [100, 60])
    keep = torch.tensor([0, 2, 3, 5]).cuda()
    q2 = alone.add([2, 2], tuple(t[keep] for t in qkv))
    o2 = alone.attend(q2, [2, 2])
    tol = 2 * torch.finfo(s.cache.dtype).eps * float(qkv[2].abs().max()) + 1e-4
    assert float((o[keep] - o2).abs().max()) <= tol
    sums = torch.zeros(2, H, 18 * PAGE, device="cuda")
    lens = torch.tensor(alone.lens, dtype=torch.int32).cuda()
    Q.attention_paged(q2[1::2], alone.cache, alone.table, lens, D ** -0.5, weights=sums)
    kept, new = Q.evict_select(sums, lens, 50, recent=8, sinks=2)
    Q.cache_compact(alone.cache, alone.table, lens, kept, new, weights=sums)
    alone.lens = new.tolist()
    step = alone.new([1, 1], 5)
    assert bool(alone.attend(alone.add([1, 1], step, torch.tensor([102, 62]).cuda()), [1, 1]).isfinite().all())
    assert Q.device_status() == 0


@pytest.mark.parametrize("kind", ["bf16", "lzs"])
def test_many_tiles_of_full_rows(Q, kind):
    """A whole tile of rows over so many keys that a CTA takes several: both warpgroups in turn, and from block to block."""
    seqs = [(12000, 64), (700, 64), (130, 64), (9000, 1)]
    Case(Q, kind, 128, 2, 2, 64, seqs, seed=3).run(Q, tree=_trees(seqs, 2))
    Case(Q, kind, 192, 2, 2, 64, [(9000, 200), (300, 200)], seed=4).run(Q)


def test_pages_shared_by_heads_and_sequences(Q):
    """Strides of 0 (one key head for all) and a prefix's pages in several tables, read only."""
    g = torch.Generator().manual_seed(1)
    one = [torch.randn(20, 16, 1, 64, generator=g).bfloat16().cuda() for _ in range(2)]
    cache = Q.PagedCache(*(t.expand(20, 16, 3, 64) for t in one), 16)
    table = torch.tensor([[4, 5, 6, 7], [4, 5, 9, 11]], dtype=torch.int32).cuda()
    lens, starts = torch.tensor([64, 50], dtype=torch.int32).cuda(), torch.tensor([0, 20, 25], dtype=torch.int32).cuda()
    q = torch.randn(25, 6, 64, generator=g).bfloat16().cuda()
    o = Q.attention_paged_tokens(q, cache, table, lens, starts, 0.125)
    dense = Q.PagedCache(*(t.expand(20, 16, 3, 64).contiguous() for t in one), 16)
    assert torch.equal(o, Q.attention_paged_tokens(q, dense, table, lens, starts, 0.125))


def test_keys_that_a_token_does_not_see(Q):
    """NaN and infinite keys of later tokens leave earlier ones as they are; their own rows and those behind are NaN."""
    c = Case(Q, "f16", 64, 1, 2, 16, [(200, 30)], seed=1)
    want = c.run(Q)
    for bad in (float("nan"), float("inf")):
        at = 170 + 20
        c.cache.k[int(c.table[0, at // 16]), at % 16] = bad
        o = Q.attention_paged_tokens(c.q.cuda(), c.cache, *c.args, 0.125)
        # (a maximum may be taken up a tile earlier: other roundings of the weights)
        near = 4 * torch.finfo(torch.float16).eps * float(c.v[0].abs().max())
        assert float((o[:20] - want[:20]).abs().max()) <= near and not bool(o[20:].isfinite().any())


def test_many_sequences(Q):
    """More sequences than CTAs, most with nothing new."""
    seqs = [(20 + i % 50, 0 if i % 3 else 1 + i % 7) for i in range(400)]
    Case(Q, "f16", 64, 1, 1, 16, seqs, seed=1).run(Q)
    Case(Q, "f16", 64, 1, 2, 16, [(n + 90, m * 13) for n, m in seqs[:60]], seed=1).run(Q)


def test_another_stream_with_its_own_memory(Q):
    c = Case(Q, "bf16", 128, 2, 2, 16, [(500, 100)], seed=1)
    q, s = c.q.cuda(), torch.cuda.Stream()
    torch.cuda.synchronize()
    o = Q.attention_paged_tokens(q, c.cache, *c.args, 128 ** -0.5, stream=s)
    s.synchronize()
    c.check(o, 128 ** -0.5)
