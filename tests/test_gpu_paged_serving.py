"""The paged cache's operators as a server uses them together: prompts
appended, tokens decoded with their weights summed, caches evicted and decoded
on; the same in a captured graph and on other streams."""
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


B, H, GROUP, D, PAGE = 3, 2, 4, 128, 16


class Server:
    """A few sequences over one cache, driven by the package's calls."""

    def __init__(self, Q, store, seed=0):
        self.Q = Q
        g = torch.Generator().manual_seed(seed)
        pages = 40
        kw = dict(params=Q.Params(group_s=16)) if store == "lzs" else dict(dtype=torch.bfloat16)
        self.cache = Q.empty_paged_cache(pages, PAGE, H, D, **kw)
        self.dtype = self.cache.dtype
        order = torch.randperm(pages, generator=g, dtype=torch.int32)
        self.table = order[:B * 12].view(B, 12).contiguous().cuda()
        self.freqs, self.scale = Q.rope_frequencies(D, base=500000.0, scaling="yarn", factor=4.0, original_length=4096)
        self.weights = torch.zeros(B, H, 12 * PAGE, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.positions = torch.zeros(B, dtype=torch.int64, device="cuda")

    def slots(self, b, t):
        return self.table.long()[b, t // PAGE] * PAGE + t % PAGE

    def prompt(self, b, k, v):
        n = k.shape[0]
        t = torch.arange(n, device="cuda")
        self.Q.paged_append(self.cache, k, v, self.slots(b, t), positions=t, freqs=self.freqs, rope_scale=self.scale)
        self.lens[b], self.positions[b] = n, n

    def step(self, q, k, v):
        """One token for every sequence; everything on the device, so that it can be captured."""
        Q = self.Q
        rows = torch.arange(B, device="cuda")
        q = Q.rope(q, self.positions, self.freqs, scale=self.scale)
        Q.paged_append(self.cache, k, v, self.slots(rows, self.lens.long()), positions=self.positions, freqs=self.freqs,
                       rope_scale=self.scale)
        self.lens += 1
        self.positions += 1
        return Q.attention_paged(q, self.cache, self.table, self.lens, D ** -0.5, out_dtype=torch.float32,
                                 weights=self.weights)

    def evict(self, budget):
        kept, new = self.Q.evict_select(self.weights, self.lens, budget, recent=8, sinks=2)
        self.Q.cache_compact(self.cache, self.table, self.lens, kept, new, weights=self.weights)
        self.lens.copy_(new)
        return kept


def _inputs(dtype, prompts, steps, seed=1):
    g = torch.Generator().manual_seed(seed)
    pr = [tuple(torch.randn(n, H, D, generator=g).to(dtype).cuda() for _ in range(2)) for n in prompts]
    st = [(torch.randn(B, H * GROUP, D, generator=g).to(dtype).cuda(),
           torch.randn(B, H, D, generator=g).to(dtype).cuda(), torch.randn(B, H, D, generator=g).to(dtype).cuda())
          for _ in range(steps)]
    return pr, st


@pytest.mark.parametrize("store", ["bf16", "lzs"])
def test_prompt_decode_evict_decode(Q, store):
    s = Server(Q, store)
    prompts, steps = _inputs(s.dtype, [100, 37, 150], 12)
    for b, (k, v) in enumerate(prompts):
        s.prompt(b, k, v)
    sums = torch.zeros(B, H, 12 * PAGE, dtype=torch.float64)
    slack = torch.zeros_like(sums)
    for i, (q, k, v) in enumerate(steps):
        pos = s.positions.clone()
        o = s.step(q, k, v)
        kh, vh = R.held(s.cache)
        qr = Q.rope(q, pos, s.freqs, scale=s.scale).cpu()
        ref, add, mag, pv = R.attention(qr, kh, vh, s.table.cpu(), s.lens.cpu(), D ** -0.5)
        bound, w_rel = R.attention_bounds(mag, pv, ref, add, int(s.lens.max()), D, GROUP, torch.float32, 17,
                                          float(vh.nan_to_num(0, 0, 0).abs().max()))
        assert bool(((o.cpu().double() - ref).abs() <= bound).all())
        sums += add
        slack = slack + add * w_rel[..., None] + sums * 2.0 ** -24
        assert bool(((s.weights.cpu().double() - sums).abs() <= slack).all())
        if i in (4, 8):
            before = R.held(s.cache)
            w_before, len_before = s.weights.cpu(), s.lens.cpu()
            kept = s.evict(64).cpu()
            want, new = R.evict(w_before, len_before, 64, 8, 2)
            assert torch.equal(kept, want) and torch.equal(s.lens.cpu(), new)
            after = R.held(s.cache)
            for x, y in zip(before, after):
                for b in range(B):
                    for h in range(H):
                        src = kept[b, h, :int(new[b])].long()
                        j = torch.arange(len(src))
                        t = s.table.cpu()[b].long()
                        assert torch.equal(y[t[j // PAGE], j % PAGE, h], x[t[src // PAGE], src % PAGE, h])
            # the reference's sums follow the rows
            for b in range(B):
                n, m = int(len_before[b]), int(new[b])
                for x in (sums, slack):
                    x[b, :, :m] = torch.stack([x[b, h, kept[b, h, :m].long()] for h in range(H)])
                    x[b, :, m:n] = 0
    assert Q.device_status() == 0


@pytest.mark.parametrize("store", ["bf16", "lzs"])
def test_captured_steps_give_the_same(Q, store):
    """A captured step replayed over changing inputs, lengths and positions equals the eager one bit for bit; two
    graphs of it, each with its own workspaces, take turns."""
    prompts, steps = _inputs(torch.float16 if store == "lzs" else torch.bfloat16, [100, 37, 60], 8, seed=2)

    def start():
        s = Server(Q, store)
        for b, (k, v) in enumerate(prompts):
            s.prompt(b, k, v)
        return s

    eager = start()
    want = [eager.step(*x).clone() for x in steps]
    s = start()
    held = tuple(x.clone() for x in steps[0])
    saved = [x.clone() for x in (s.lens, s.positions, s.weights)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(*held)                                    # warm-up: the same token is written again below
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = s.step(*held)
        graphs.append((g, out))
    for x, y in zip((s.lens, s.positions, s.weights), saved):
        x.copy_(y)
    for i, x in enumerate(steps):
        for a, b in zip(held, x):
            a.copy_(b)
        g, out = graphs[i % 2]
        g.replay()
        assert torch.equal(out, want[i]), i
    assert torch.equal(s.weights, eager.weights) and Q.device_status() == 0


def test_two_streams_at_once(Q):
    """Two servers on two streams, steps interleaved without waiting, equal each by itself."""
    prompts, steps = _inputs(torch.float16, [100, 37, 150], 6, seed=3)

    def start(seed):
        s = Server(Q, "lzs", seed)
        for b, (k, v) in enumerate(prompts):
            s.prompt(b, k, v)
        return s

    alone = [start(i) for i in range(2)]
    want = [[s.step(*x).clone() for x in steps] for s in alone]
    both = [start(i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    got = [[], []]
    for x in steps:
        for i, (s, st) in enumerate(zip(both, streams)):
            with torch.cuda.stream(st):
                got[i].append(s.step(*x))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))
    assert Q.device_status() == 0


def test_explicit_stream_argument(Q):
    """`stream=` runs the call there, not on the current stream."""
    s = Server(Q, "bf16")
    prompts, steps = _inputs(s.dtype, [100, 37, 150], 1, seed=4)
    for b, (k, v) in enumerate(prompts):
        s.prompt(b, k, v)
    q = steps[0][0]
    want = Q.attention_paged(q, s.cache, s.table, s.lens, 0.1)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, ws = torch.empty_like(want), torch.empty(Q.attention_paged_workspace_size(s.cache, B, H * GROUP, 12 * PAGE),
                                                  dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    Q.attention_paged(q, s.cache, s.table, s.lens, 0.1, out=out, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
