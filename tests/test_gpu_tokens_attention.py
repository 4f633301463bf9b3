"""Attention of several new tokens per sequence over a paged cache, against the
definition in 64 bits."""
import math
import random

import pytest

import tokens_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "lzs": torch.float16}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _encoded(g, rows, D, gs):
    """Codes, FLAGs and scales, and what they stand for."""
    c = torch.randint(-8, 8, (rows, D), generator=g)
    f = torch.randint(0, 5, (rows, D // gs), generator=g)
    s = (torch.rand((rows, D // 64), generator=g) * 0.03 + 0.001).half()
    codes = ((c[:, 0::2] & 15) | ((c[:, 1::2] & 15) << 4)).to(torch.uint8)
    value = (c << f.repeat_interleave(gs, 1)).double() * s.double().repeat_interleave(64, 1)
    return codes, f.to(torch.uint8), s, value.half()


class Case:
    """Sequences (cached, new) over shuffled pages; every place that no sequence's token has is NaN."""

    def __init__(self, Q, kind, D, H, G, page, seqs, gs=16, seed=0, heads_first=False, order=None):
        g = torch.Generator().manual_seed(seed)
        self.seqs, self.H, self.G, self.D, self.page, self.kind = seqs, H, G, D, page, kind
        dtype = DTYPES[kind]
        need = [-(-n // page) for n, _ in seqs]
        pages = sum(need) + 2
        perm = torch.randperm(pages, generator=g).tolist()
        self.table = torch.full((len(seqs), max(need + [1]) + 1), -1, dtype=torch.int32)
        self.k, self.v = [], []
        held, i = torch.zeros((pages, page), dtype=torch.bool), 0
        where = []
        for b, (n, _) in enumerate(seqs):
            mine = perm[i:i + need[b]]
            i += need[b]
            self.table[b, :need[b]] = torch.tensor(mine, dtype=torch.int32)
            t = torch.arange(n)
            at = torch.tensor(mine, dtype=torch.int64)[t // page] if n else t
            held[at, t % page] = True
            where.append((at, t % page))
        if kind == "lzs":
            rows = pages * H * page
            sides = []
            for side in range(2):
                codes, f, s, value = _encoded(g, rows, D, gs)
                bad = ~held[:, None].expand(pages, H, page).reshape(-1)
                s[bad] = float("nan")
                p = Q.Params(group_s=gs)
                sides.append(Q.Encoded(codes.cuda(), f.cuda(), s.cuda(), None, None, rows, D, p))
                value = value.view(pages, H, page, D).transpose(1, 2)
                (self.v if side else self.k).extend(value[at, slot] for at, slot in where)
            self.cache = Q.PagedCache(*sides, page, H)
        else:
            pools = []
            for side in range(2):
                x = torch.randn((pages, page, H, D), generator=g).to(dtype)
                (self.v if side else self.k).extend(x[at, slot] for at, slot in where)
                x[~held] = float("nan")
                x = x.cuda()
                pools.append(x.transpose(1, 2).contiguous().transpose(1, 2) if heads_first else x)
            self.cache = Q.PagedCache(*pools, page)
        self.starts = [0]
        for _, m in seqs:
            self.starts.append(self.starts[-1] + m)
        self.q = torch.randn((self.starts[-1], H * G, D), generator=g).to(dtype)
        self.args = (self.table.cuda(), torch.tensor([n for n, _ in seqs], dtype=torch.int32).cuda(),
                     torch.tensor(self.starts, dtype=torch.int32).cuda())

    def check(self, o, scale, tree=None, window=0, prefix=None, cap=0.0, slopes=None):
        dtype = DTYPES[self.kind]
        for b, (n, m) in enumerate(self.seqs):
            s0 = self.starts[b]
            t = None if tree is None else tree[s0:s0 + m]
            pre = 0 if prefix is None else prefix[b]
            mask = R.seen(n, m, t, window, pre)
            pos, place = R.places(n, m, t)
            ref, bound = R.attention(self.q[s0:s0 + m], self.k[b], self.v[b], scale, mask, dtype,
                                     torch.tensor(pos), torch.tensor(place), cap, slopes)
            got = o[s0:s0 + m].cpu().double()
            off = (got - ref).abs() - R.rounded(bound, ref, o.dtype)
            assert bool((off <= 0).all()), (b, n, m, float(off.max()), float((got - ref).abs().max()))

    def run(self, Q, scale=None, tree=None, window=0, prefix=None, cap=0.0, slopes=None, **how):
        scale = self.D ** -0.5 if scale is None else scale
        signed = None if tree is None else torch.tensor([t - (1 << 64) if t >> 63 else t for t in tree]).cuda()
        o = Q.attention_paged_tokens(self.q.cuda(), self.cache, *self.args, scale, tree=signed, window=window, cap=cap,
                                     prefix_lens=None if prefix is None else torch.tensor(prefix, dtype=torch.int32).cuda(),
                                     slopes=None if slopes is None else slopes.cuda(), **how)
        self.check(o, scale, tree, window, prefix, cap, slopes)
        assert Q.device_status() == 0
        return o


def _trees(seqs, seed):
    rng = random.Random(seed)
    out = []
    for _, m in seqs:
        masks = []
        for j in range(m):
            parent = rng.randrange(-1, j) if j else -1
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << j)
        out += masks
    return out


# lengths around a tile of keys, one token, no context, nothing new
RAGGED = [(1, 1), (130, 3), (128, 128), (257, 129), (5, 0), (300, 40), (64, 64)]


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("H,G", [(2, 1), (1, 4), (2, 3)])
def test_causal(Q, kind, D, H, G):
    Case(Q, kind, D, H, G, 16, RAGGED, seed=D + G).run(Q)


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("page", [1, 2, 8, 64, 256, 4096])
def test_page_sizes(Q, kind, page):
    Case(Q, kind, 64, 2, 2, page, [(200, 70), (131, 1), (70, 70)], seed=page).run(Q)


@pytest.mark.parametrize("gs", [8, 16, 32, 64])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_subgroups(Q, gs, D):
    Case(Q, "lzs", D, 2, 2, 32, [(200, 70), (131, 1)], gs=gs, seed=gs).run(Q)


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("window", [1, 20, 64, 200])
def test_window(Q, kind, D, window):
    Case(Q, kind, D, 2, 3, 16, [(400, 150), (30, 30), (500, 2)], seed=window).run(Q, window=window)


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("window", [0, 40])
def test_prefix(Q, kind, window):
    seqs = [(600, 150), (30, 30), (500, 2), (7, 3)]
    Case(Q, kind, 128, 2, 2, 16, seqs, seed=3).run(Q, window=window, prefix=[130, 30, 0, 5])


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 256])
@pytest.mark.parametrize("cap,sloped", [(5.0, False), (0.0, True), (30.0, True)])
def test_cap_and_slopes(Q, kind, D, cap, sloped):
    c = Case(Q, kind, D, 2, 3, 16, [(300, 140), (40, 3)], seed=5)
    slopes = 2.0 ** -torch.arange(1, 7, dtype=torch.float32) if sloped else None
    c.run(Q, cap=cap, slopes=slopes)


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(2, 1), (1, 8), (2, 3)])
def test_tree(Q, kind, D, H, G):
    seqs = [(140, 12), (64, 64), (300, 61), (9, 1), (12, 0), (1, 1)]
    Case(Q, kind, D, H, G, 16, seqs, seed=D + G).run(Q, tree=_trees(seqs, G))


@pytest.mark.parametrize("window", [1, 3, 30, 100])
def test_tree_with_everything(Q, window):
    seqs = [(140, 12), (64, 64), (300, 61), (20, 20)]
    Case(Q, "bf16", 128, 2, 3, 16, seqs, seed=window).run(Q, tree=_trees(seqs, 3), window=window, prefix=[3, 0, 270, 20],
                                                         cap=20.0, slopes=2.0 ** -torch.arange(1, 7, dtype=torch.float32))


def test_masks_of_any_bits(Q):
    """Bits of later tokens, none at all (nothing cached before: nothing seen, zeros), and bits behind the last token."""
    seqs = [(5, 5), (70, 6), (64, 64)]
    rng = random.Random(1)
    tree = [0, 1 << 4, 31, ~0 & (2 ** 64 - 1), 1 << 63] + [0, 1, 2, 63, 1 << 60, 9] + [rng.getrandbits(64) for _ in range(64)]
    c = Case(Q, "f16", 64, 2, 2, 8, seqs, seed=2)
    o = c.run(Q, tree=tree)
    assert bool((o[0] == 0).all()) and bool((o[4] == 0).all())


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D,G", [(64, 2), (128, 1), (128, 8), (192, 2), (256, 3)])
def test_cut_tiles_are_joined(Q, kind, D, G):
    """Few rows over long contexts, and blocks that take several CTAs in part and in whole."""
    Case(Q, kind, D, 1, G, 64, [(5000, 9)], seed=D).run(Q, tree=_trees([(5000, 9)], 1))
    Case(Q, kind, D, 1, G, 64, [(3001, 333), (700, 5), (2000, 130)], seed=D).run(Q)


@pytest.mark.parametrize("out", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_result_types(Q, kind, out):
    for seqs in ([(200, 70)], [(4000, 3)]):
        o = Case(Q, kind, 128, 2, 2, 16, seqs, seed=9).run(Q, out_dtype=out)
        assert o.dtype == out


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(Q, scale):
    """None, negative, and so large that maxima rise from tile to tile."""
    for kind in ("f16", "bf16"):
        Case(Q, kind, 64, 2, 2, 16, [(700, 70), (64, 64)], seed=11).run(Q, scale=scale)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_rising_scores(Q, kind):
    """The last keys weigh most: what came before is rescaled, to nothing."""
    c = Case(Q, kind, 128, 1, 1, 16, [(1000, 5)], seed=1)
    c.q[:] = 1.0
    up = torch.arange(1000, dtype=torch.float32)[:, None, None] / 100
    c.k[0] = (c.k[0].float() * 0.01 + up).to(c.q.dtype)
    flat = torch.arange(1000)
    pool = c.cache.k
    pool[c.table[0][flat // 16].long().cuda(), (flat % 16).cuda()] = c.k[0].cuda()
    c.run(Q)


def test_strides(Q):
    """Queries out of a fused projection, a [pages, heads, slots, dim] pool, a table out of a larger one."""
    for kind in ("f16", "bf16"):
        c = Case(Q, kind, 64, 2, 3, 16, RAGGED, seed=4, heads_first=True)
        fused = torch.randn((c.q.shape[0], 10, 64)).to(c.q.dtype).cuda()
        fused[:, 2:8] = c.q.cuda()
        wide = torch.full((c.table.shape[0], c.table.shape[1] + 5), -1, dtype=torch.int32).cuda()
        wide[:, :c.table.shape[1]] = c.args[0]
        o = Q.attention_paged_tokens(fused[:, 2:8], c.cache, wide[:, :c.table.shape[1]], *c.args[1:], 0.125)
        c.check(o, 0.125)


def test_rows_of_no_sequence_stay(Q):
    c = Case(Q, "bf16", 64, 2, 2, 16, [(40, 3), (200, 130)], seed=6)
    T = c.starts[-1]
    q = torch.full((T + 9, 4, 64), float("nan"), dtype=torch.bfloat16).cuda()
    q[4:4 + T] = c.q.cuda()
    out = torch.full((T + 9, 4, 64), 7.0, dtype=torch.float32).cuda()
    Q.attention_paged_tokens(q, c.cache, c.args[0], c.args[1], c.args[2] + 4, 0.125, out=out)
    c.check(out[4:4 + T], 0.125)
    assert bool((out[:4] == 7).all()) and bool((out[4 + T:] == 7).all())


@pytest.mark.parametrize("kind", ["f16", "lzs"])
def test_one_new_token_agrees_with_attention_paged(Q, kind):
    seqs = [(n, 1) for n in (1, 17, 128, 1000, 3000)]
    c = Case(Q, kind, 128, 2, 4, 16, seqs, seed=8)
    a = c.run(Q, out_dtype=torch.float32)
    b = Q.attention_paged(c.q.cuda(), c.cache, c.args[0], c.args[1], 128 ** -0.5, out_dtype=torch.float32)
    # both within the bound of the definition; attention_paged() does not round the weights
    c.check(b, 128 ** -0.5)
    assert float((a - b).abs().max()) < 0.02


def test_bounds_of_the_caller(Q):
    """Tight max_len and max_new plan less and answer the same; a workspace of the caller's."""
    seqs = [(300, 9), (77, 5)]
    c = Case(Q, "f16", 128, 2, 2, 16, seqs, seed=3)
    c.run(Q, max_len=300, max_new=9)
    size = Q.attention_paged_tokens_workspace_size(c.cache, 14, 2, 4, 300, 9)
    c.run(Q, max_len=300, max_new=9, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
    with pytest.raises(Q.QuartzError):
        c.run(Q, max_len=300, max_new=9, workspace=torch.empty(size - 256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("what", ["len", "short", "start", "order", "many", "page"])
def test_bad_numbers_on_the_device_are_reported(Q, what):
    seqs = [(40, 3), (200, 130), (50, 2)]
    c = Case(Q, "f16", 64, 2, 2, 16, seqs, seed=6)
    table, lens, starts = (t.clone() for t in c.args)
    how = {}
    if what == "len":
        lens[1] = table.shape[1] * 16 + 1
    elif what == "short":
        lens[1] = 129
    elif what == "start":
        starts[3] = c.starts[-1] + 1
    elif what == "order":
        starts[2] = starts[1] - 1
    elif what == "many":
        how = dict(max_new=100)
    else:
        table[1, 3] = 1 << 20
    o = Q.attention_paged_tokens(c.q.cuda(), c.cache, table, lens, starts, 0.125, **how)
    assert Q.device_status() == 7 and Q.device_status() == 0
    first = c.seqs[:1]
    c.seqs = first
    c.check(o, 0.125)


def test_captured_and_replayed(Q):
    """Lengths, starts and pages are the device's: a graph follows them."""
    a = Case(Q, "bf16", 128, 2, 2, 16, [(300, 20), (500, 3), (64, 17)], seed=1)
    b = Case(Q, "bf16", 128, 2, 2, 16, [(30, 1), (490, 30), (64, 9)], seed=2)
    pools = [torch.empty_like(a.cache.k), torch.empty_like(a.cache.v)]
    cache = Q.PagedCache(*pools, 16)
    q = torch.zeros_like(a.q).cuda()
    args = [torch.zeros_like(t) for t in a.args]
    out = torch.zeros(q.shape, dtype=torch.float32, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        Q.attention_paged_tokens(q, cache, *args, 0.1, max_new=32, out=out)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Q.attention_paged_tokens(q, cache, *args, 0.1, max_new=32, out=out)
    for c in (a, b, a):
        for pool, x in zip(pools, (c.cache.k, c.cache.v)):
            pool[:x.shape[0]] = x[:pool.shape[0]]
        if c.table.shape[1] > args[0].shape[1] or c.cache.num_pages > cache.num_pages:
            pytest.skip("the cases are chosen to fit")
        args[0].fill_(-1)
        args[0][:, :c.table.shape[1]] = c.args[0]
        args[1].copy_(c.args[1])
        args[2].copy_(c.args[2])
        q.zero_()
        q[:c.q.shape[0]] = c.q.cuda()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, 0.1)
    assert Q.device_status() == 0


def test_two_streams_at_once_and_the_same_twice(Q):
    cases = [Case(Q, "bf16", 128, 2, 4, 16, [(2000, 200)], seed=i) for i in range(2)]
    qs = [c.q.cuda() for c in cases]
    want = [Q.attention_paged_tokens(q, c.cache, *c.args, 0.1) for q, c in zip(qs, cases)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(5):
        for i, (q, c) in enumerate(zip(qs, cases)):
            got[i].append(Q.attention_paged_tokens(q, c.cache, *c.args, 0.1, stream=streams[i]))
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(w, x) for x in many)


def test_mismatched_arguments_are_refused(Q):
    c = Case(Q, "f16", 64, 2, 2, 16, [(40, 3), (50, 2)], seed=1)
    q, (table, lens, starts) = c.q.cuda(), c.args
    tree = torch.ones(5, dtype=torch.int64, device="cuda")
    for args, how in [((q.bfloat16(), c.cache, table, lens, starts, 1.0), {}), ((q[:, :3], c.cache, table, lens, starts, 1.0), {}),
                      ((q[..., :32], c.cache, table, lens, starts, 1.0), {}), ((q, c.cache, table, lens, starts[:2], 1.0), {}),
                      ((q, c.cache, table, lens[:1], starts, 1.0), {}), ((q, c.cache, table, lens.long(), starts, 1.0), {}),
                      ((q, c.cache, table, lens, starts, 1.0), dict(max_len=10 ** 6)),
                      ((q, c.cache, table, lens, starts, 1.0), dict(max_new=-1)),
                      ((q, c.cache, table, lens, starts, 1.0), dict(tree=tree[:4])),
                      ((q, c.cache, table, lens, starts, 1.0), dict(tree=tree.int())),
                      ((q, c.cache, table, lens, starts, 1.0), dict(prefix_lens=lens[:1])),
                      ((q, c.cache, table, lens, starts, 1.0), dict(slopes=torch.ones(3, device="cuda"))),
                      ((q, c.cache, table, lens, starts, 1.0), dict(out=torch.empty((5, 4, 32), device="cuda"))),
                      ((q, c.cache, table, lens, starts, 1.0), dict(out_dtype=torch.float64))]:
        with pytest.raises(ValueError):
            Q.attention_paged_tokens(*args, **how)
    for how in (dict(window=-1), dict(cap=-1.0), dict(cap=math.inf), dict(cap=math.nan)):
        with pytest.raises(Q.QuartzError):
            Q.attention_paged_tokens(q, c.cache, table, lens, starts, 1.0, **how)
    assert Q.attention_paged_tokens(q[:0], c.cache, table, lens, starts * 0, 1.0).shape == (0, 4, 64)
