"""The norm of each head with the rotation, its gradient, and rotary positions of
several axes, against the definitions in 64 bits."""
import pytest

import tokens_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _x(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


def _places(T, axes, seed):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-3, 1 << 17, (axes, T), generator=g)
    p[:, 0] = 0
    return p


def _rope(r, axes):
    """freqs, and each pair's axis (in no order)."""
    n = r // 2
    return 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n), [(7 * i + i // 3) % axes for i in range(n)]


# (tokens, heads, dim, rotary, axes): whole and partial heads, widths that no vector divides, one token, one pair, many heads
AXES = [(1, 1, 64, 64, 2), (3, 5, 128, 128, 3), (7, 2, 96, 64, 3), (5, 3, 80, 40, 2), (2, 33, 256, 256, 3), (4, 1, 6, 2, 1),
        (3, 2, 37, 36, 4), (130, 9, 72, 72, 2), (2, 1, 255, 2, 2)]


@pytest.mark.parametrize("T,H,D,r,axes", AXES)
@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("interleaved,backward", [(False, False), (True, False), (False, True), (True, True)])
def test_rope_axes(Q, T, H, D, r, axes, dt, interleaved, backward):
    dtype = DTYPES[dt]
    x, pos, (freqs, axis) = _x((T, H, D), dtype, 1), _places(T, axes, 2), _rope(r, axes)
    y = Q.rope_axes(x.cuda(), pos.cuda(), freqs.cuda(), torch.tensor(axis, dtype=torch.int32).cuda(),
                    interleaved=interleaved, scale=1.25, backward=backward).cpu()
    ref = R.rope_axes(x, pos, freqs, axis, interleaved, 1.25, backward)
    bound = R.turn_bound(x.double().abs(), 0.0, pos, freqs, axis, interleaved, 1.25)
    assert y.dtype == dtype and bool(((y.double() - ref).abs() <= R.rounded(bound, ref, dtype)).all())
    assert torch.equal(y[..., r:], x[..., r:])


@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
def test_one_axis_is_rope(Q, dt, interleaved):
    """Pairs of one axis only: the bits of rope()."""
    x, pos = _x((37, 5, 96), DTYPES[dt], 3).cuda(), _places(37, 2, 4).cuda()
    freqs, _ = _rope(64, 1)
    axis = torch.ones(32, dtype=torch.int32, device="cuda")
    y = Q.rope_axes(x, pos, freqs.cuda(), axis, interleaved=interleaved)
    assert torch.equal(y, Q.rope(x, pos[1], freqs.cuda(), interleaved=interleaved))


def test_an_axis_out_of_range_is_reported(Q):
    x, pos = _x((3, 2, 64), torch.float16, 3).cuda(), _places(3, 2, 4).cuda()
    freqs, _ = _rope(64, 2)
    for bad in (-1, 2):
        axis = torch.zeros(32, dtype=torch.int32)
        axis[5] = bad
        Q.rope_axes(x, pos, freqs.cuda(), axis.cuda())
        assert Q.device_status() == 7
    assert Q.device_status() == 0


# (tokens, q heads, k heads, dim, rotary, axes): 0 axes: one, as a vector of positions; rotary 0: none
NORMS = [(1, 1, 1, 64, 64, 0), (5, 4, 2, 128, 128, 0), (3, 24, 24, 128, 128, 3), (7, 5, 1, 96, 64, 2), (9, 3, 2, 80, 0, 0),
         (2, 33, 7, 256, 256, 0), (4, 1, 1, 6, 2, 1), (3, 2, 1, 37, 36, 0), (150, 8, 2, 72, 72, 2), (1, 3, 1, 2, 2, 0),
         (2, 2, 2, 255, 2, 0), (6, 2, 0, 64, 64, 0)]


def _norm_case(T, Hq, Hk, D, r, axes, dtype, wt):
    q, k = _x((T, Hq, D), dtype, 1) * 3, (_x((T, Hk, D), dtype, 2) if Hk else None)
    if T > 1:
        q[1, 0] = 0  # a head of nothing: eps alone
    w_dtype = {"same": dtype, "f32": torch.float32, "none": None}[wt]
    ws = [None if w_dtype is None or x is None else (1 + 0.2 * _x((D,), torch.float32, s)).to(w_dtype)
          for x, s in ((q, 3), (k, 4))]
    pos = freqs = axis = None
    if r:
        freqs, axis = _rope(r, max(axes, 1))
        pos = _places(T, max(axes, 1), 5)
        if axes == 0:
            pos, axis = pos[0], None
    return q, k, ws, pos, freqs, axis


def _cuda(t, kind=None):
    return None if t is None else torch.as_tensor(t, dtype=kind).cuda()


@pytest.mark.parametrize("T,Hq,Hk,D,r,axes", NORMS)
@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("interleaved,wt", [(False, "same"), (True, "f32"), (False, "none")])
def test_norm_and_gradient(Q, T, Hq, Hk, D, r, axes, dt, interleaved, wt):
    dtype = DTYPES[dt]
    q, k, ws, pos, freqs, axis = _norm_case(T, Hq, Hk, D, r, axes, dtype, wt)
    eps, scale = 1e-5, 1.25 if r else 1.0
    how = dict(eps=eps, pair_axis=_cuda(axis, torch.int32), interleaved=interleaved, scale=scale)
    args = (_cuda(q), _cuda(k), _cuda(ws[0]), _cuda(ws[1]), _cuda(pos), _cuda(freqs))
    ys = Q.qk_norm_rope(*args, **how)
    dys = [None if x is None else _x(x.shape, dtype, s) for x, s in ((q, 6), (k, 7))]
    grads = Q.qk_norm_rope_backward(_cuda(dys[0]), _cuda(dys[1]), *args, **how)
    for i, x in enumerate((q, k)):
        if x is None:
            assert ys[i] is None and grads[i] is None and grads[2 + i] is None
            continue
        ref, bound = R.norm(x, ws[i], eps, pos, freqs, axis, interleaved, scale)
        assert ys[i].dtype == dtype
        assert bool(((ys[i].cpu().double() - ref).abs() <= R.rounded(bound, ref, dtype)).all())
        dx, dw, e_dx, e_dw = R.norm_grad(x, ws[i], dys[i], eps, pos, freqs, axis, interleaved, scale)
        assert bool(((grads[i].cpu().double() - dx).abs() <= R.rounded(e_dx, dx, dtype)).all())
        if ws[i] is None:
            assert grads[2 + i] is None
        else:
            got = grads[2 + i].cpu()
            assert got.dtype == ws[i].dtype
            assert bool(((got.double() - dw).abs() <= R.rounded(e_dw, dw, got.dtype)).all())
    assert Q.device_status() == 0


@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_views_of_a_projection(Q, dt, offset):
    """Queries and keys side by side, at an address that the type, 8 or 16 bytes align; in place; the values stay."""
    dtype, T, Hq, Hk, D = DTYPES[dt], 11, 4, 2, 64
    flat = _x((T * (Hq + 2 * Hk) * D + 16,), dtype, 1).cuda()
    x = flat[offset:offset + T * (Hq + 2 * Hk) * D].view(T, Hq + 2 * Hk, D)
    before, head = x.clone(), flat[:offset].clone()
    w, pos, (freqs, _) = _x((D,), dtype, 2).cuda(), _places(T, 1, 3)[0].cuda(), _rope(D, 1)
    q, k = x[:, :Hq], x[:, Hq:Hq + Hk]
    want = Q.qk_norm_rope(q.contiguous(), k.contiguous(), w, w, pos, freqs.cuda())
    dy = [_x(t.shape, dtype, 4).cuda() for t in (q, k)]
    g1 = Q.qk_norm_rope_backward(*dy, q, k, w, w, pos, freqs.cuda())
    g2 = Q.qk_norm_rope_backward(*dy, q.contiguous(), k.contiguous(), w, w, pos, freqs.cuda())
    assert Q.qk_norm_rope(q, k, w, w, pos, freqs.cuda(), out=(q, k))[0] is q
    # another vector width sums the squares in another order: a step of the type at most, as each is within half a step
    # and a few of binary32's
    for a, b in zip((q, k), want):
        ulp = torch.finfo(dtype).eps * b.abs().double() + 2.0 ** -20
        assert bool(((a.double() - b.double()).abs() <= (1 if dtype != torch.float32 else 64) * ulp).all())
    assert torch.equal(x[:, Hq + Hk:], before[:, Hq + Hk:]) and torch.equal(flat[:offset], head)
    for a, b in zip(g1, g2):
        scale = b.double().abs().max()
        assert bool(((a.double() - b.double()).abs() <= 2 * torch.finfo(dtype).eps * scale + 2.0 ** -16 * scale).all())


def test_many_rows_take_the_same_values(Q):
    """Blocks of many tokens give the values of one token alone; sums are the same on every call."""
    T, Hq, Hk, D = 4099, 6, 2, 128
    q, k = _x((T, Hq, D), torch.bfloat16, 1).cuda(), _x((T, Hk, D), torch.bfloat16, 2).cuda()
    w = (1 + 0.1 * _x((D,), torch.float32, 3)).cuda()
    pos, freqs = _places(T, 1, 4)[0].cuda(), _rope(D, 1)[0].cuda()
    yq, yk = Q.qk_norm_rope(q, k, w, w, pos, freqs)
    g = Q.qk_norm_rope_backward(yq, yk, q, k, w, w, pos, freqs)
    for t in (0, 15, 16, 2048, T - 1):
        one = slice(t, t + 1)
        y1 = Q.qk_norm_rope(q[one], k[one], w, w, pos[one], freqs)
        assert torch.equal(yq[one], y1[0]) and torch.equal(yk[one], y1[1])
        g1 = Q.qk_norm_rope_backward(yq[one], yk[one], q[one], k[one], w, w, pos[one], freqs)
        assert torch.equal(g[0][one], g1[0]) and torch.equal(g[1][one], g1[1])
    again = Q.qk_norm_rope_backward(yq, yk, q, k, w, w, pos, freqs)
    assert all(torch.equal(a, b) for a, b in zip(g, again))
    dw = R.norm_grad(q.cpu(), w.cpu(), yq.cpu(), 1e-6, pos.cpu(), freqs.cpu(), None, False, 1.0)
    assert bool(((g[2].cpu().double() - dw[1]).abs() <= R.rounded(dw[3], dw[1], torch.float32)).all())


def test_no_tokens_and_no_heads(Q):
    e, w = torch.empty((0, 2, 64), device="cuda"), torch.ones(64, device="cuda")
    assert Q.qk_norm_rope(e, e, w, w)[0].shape == (0, 2, 64)
    for n in (e, torch.empty((3, 0, 64), device="cuda")):
        dq, dk, dwq, dwk = Q.qk_norm_rope_backward(n, n, n, n, w, w)
        assert dq.shape == n.shape and bool((dwq == 0).all()) and bool((dwk == 0).all())


def test_gradient_against_differences(Q):
    """Along a direction: the kernel's own results at x +- h d.  Each difference is off by what two results are off by over
    2 h, and by what the third derivative adds, which halving h in 64 bits shows (4/3 of the change, a tenth to spare)."""
    T, H, D, eps, h = 3, 2, 64, 1e-5, 2.0 ** -6
    x, w, dy, d = (_x(s, torch.float32, i) for i, s in enumerate(((T, H, D), (D,), (T, H, D), (T, H, D))))
    pos, (freqs, axis) = _places(T, 3, 9), _rope(48, 3)
    how = dict(eps=eps, pair_axis=_cuda(axis, torch.int32))
    place = (_cuda(pos), _cuda(freqs))

    def loss(x, w):
        return float((Q.qk_norm_rope(x.cuda(), None, w.cuda(), None, *place, **how)[0].cpu().double() * dy.double()).sum())

    def exact(x, w):
        return float((R.norm(x, w, eps, pos, freqs, axis, False, 1.0)[0] * dy.double()).sum())

    dx, _, dw, _ = Q.qk_norm_rope_backward(dy.cuda(), None, x.cuda(), None, w.cuda(), None, *place, **how)
    ref, bound = R.norm(x, w, eps, pos, freqs, axis, False, 1.0)
    noise = float((R.rounded(2 * bound, ref, torch.float32) * dy.double().abs()).sum()) / h
    for got, by in ((float((dx.cpu().double() * d.double()).sum()), lambda f, h: f(x + h * d, w) - f(x - h * d, w)),
                    (float((dw.cpu().double() * d[0, 0].double()).sum()),
                     lambda f, h: f(x, w + h * d[0, 0]) - f(x, w - h * d[0, 0]))):
        third = abs(by(exact, h) / (2 * h) - by(exact, h / 2) / h) * 4 / 3 * 1.1
        assert abs(by(loss, h) / (2 * h) - got) <= 2 * noise + third + 1e-5 * abs(got)


def test_as_an_autograd_function_and_in_a_graph(Q):
    """The documented way to train with it; then the same calls captured, replayed on new inputs."""
    T, Hq, Hk, D = 33, 4, 2, 64
    pos, freqs = _places(T, 1, 1)[0].cuda(), _rope(D, 1)[0].cuda()

    class NormRope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, wq, wk):
            ctx.save_for_backward(q, k, wq, wk)
            return Q.qk_norm_rope(q, k, wq, wk, pos, freqs)

        @staticmethod
        def backward(ctx, gq, gk):
            return Q.qk_norm_rope_backward(gq, gk, *ctx.saved_tensors, pos, freqs)

    def inputs(seed):
        return [_x(s, torch.bfloat16, seed + i).cuda() for i, s in enumerate(((T, Hq, D), (T, Hk, D), (D,), (D,)))]

    leaves = [t.requires_grad_(True) for t in inputs(1)]
    yq, yk = NormRope.apply(*leaves)
    (yq.float().square().sum() + yk.float().sum()).backward()
    with torch.no_grad():
        want = Q.qk_norm_rope_backward((2 * yq.float()).bfloat16(), torch.ones_like(yk), *leaves, pos, freqs)
    assert all(torch.equal(a.grad, b) for a, b in zip(leaves, want))

    static = inputs(10)
    dy = [_x((T, Hq, D), torch.bfloat16, 20).cuda(), _x((T, Hk, D), torch.bfloat16, 21).cuda()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        Q.qk_norm_rope_backward(*dy, *static, pos, freqs)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = Q.qk_norm_rope(*static, pos, freqs)
        g = Q.qk_norm_rope_backward(*dy, *static, pos, freqs)
    for seed in (30, 40):
        for t, new in zip(static, inputs(seed)):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(y + g, Q.qk_norm_rope(*static, pos, freqs) + Q.qk_norm_rope_backward(*dy, *static, pos, freqs)):
            assert torch.equal(a, b)


def test_another_stream(Q):
    """`stream`: results are written, and their memory is given, there."""
    q = _x((64, 4, 128), torch.float16, 1).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, _ = Q.qk_norm_rope(q, None, None, None, stream=s)
    s.synchronize()
    assert torch.equal(y, Q.qk_norm_rope(q, None, None, None)[0])


def test_mismatched_arguments_are_refused(Q):
    q, k, w = (torch.zeros(s, device="cuda") for s in ((3, 2, 64), (3, 1, 64), (64,)))
    pos, freqs = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    axis = torch.zeros(32, dtype=torch.int32, device="cuda")
    for args, how in [((q, k[:2], w, w), {}), ((q, k[..., :32], w, w), {}), ((q, k, w[:32], w), {}), ((q, k, w, w.half()), {}),
                      ((q, k.half(), w, w), {}), ((q, k, w, w, pos), {}), ((q, k, w, w, None, freqs), {}),
                      ((q, k, w, w, pos[:2], freqs), {}), ((q, k, w, w, pos, freqs), dict(pair_axis=axis)),
                      ((q, k, w, w, pos[None], freqs), dict(pair_axis=axis[:3])), ((q, k, w, w, pos, freqs.float()), {}),
                      ((q.double(), k, w, w), {}), ((q, k, w, w), dict(out=(q[:2], k)))]:
        with pytest.raises(ValueError):
            Q.qk_norm_rope(*args, **how)
    for dys in ((q, None), (None, k), (q[:2], k), (q.half(), k)):
        with pytest.raises(ValueError):
            Q.qk_norm_rope_backward(*dys, q, k, w, w)
    with pytest.raises(ValueError):
        Q.rope_axes(q, pos[None], freqs, None)
    with pytest.raises(ValueError):
        Q.rope_axes(q, pos, freqs, axis)
