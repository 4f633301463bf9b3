"""Rotary positions against the definition in 64 bits."""
import pytest

import paged_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _x(T, H, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, H, D, generator=g).to(dtype)


def _positions(T, seed, top=1 << 20):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(0, top, (T,), generator=g)
    p[0] = 0
    return p


# (tokens, heads, dim, rotary): whole and partial heads, widths that no vector divides, one token, many heads
SHAPES = [(1, 1, 64, 64), (3, 5, 128, 128), (7, 2, 96, 64), (5, 3, 80, 40), (2, 33, 128, 128), (4, 1, 6, 2), (3, 2, 37, 36),
          (2, 3, 1024, 512), (2, 3, 520, 512), (130, 9, 64, 32)]


@pytest.mark.parametrize("T,H,D,r", SHAPES)
@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("interleaved,backward", [(False, False), (True, False), (False, True), (True, True)])
def test_rotation(Q, T, H, D, r, dt, interleaved, backward):
    dtype = DTYPES[dt]
    x, pos = _x(T, H, D, dtype, 1), _positions(T, 2)
    freqs, _ = Q.rope_frequencies(r, base=500000.0, device="cpu")
    scale = 1.25
    y = Q.rope(x.cuda(), pos.cuda(), freqs.cuda(), interleaved=interleaved, scale=scale, backward=backward).cpu()
    ref = R.rope(x, pos, freqs, interleaved, scale, backward)
    bound = R.rope_bound(x, pos, freqs, interleaved, scale, dtype, ref)
    assert y.dtype == dtype and bool(((y.double() - ref).abs() <= bound).all())
    assert torch.equal(y[..., r:], x[..., r:])       # what is not rotated is copied


@pytest.mark.parametrize("positions", [[0, -1, -100000, 1 << 31, (1 << 31) + 12345, 131071]])
def test_far_and_negative_positions(Q, positions):
    pos = torch.tensor(positions)
    x = _x(len(positions), 2, 64, torch.float32, 3)
    freqs, _ = Q.rope_frequencies(64, device="cpu")
    y = Q.rope(x.cuda(), pos.cuda(), freqs.cuda()).cpu()
    ref = R.rope(x, pos, freqs)
    assert bool(((y.double() - ref).abs() <= R.rope_bound(x, pos, freqs, False, 1.0, torch.float32, ref)).all())


def test_many_tokens_and_heads_take_the_same_values(Q):
    """The variant for many tokens (several heads per thread) rounds as the one for few."""
    x, pos = _x(2048, 37, 128, torch.bfloat16, 4).cuda(), _positions(2048, 5).cuda()
    freqs = Q.rope_frequencies(128)[0]
    y = Q.rope(x, pos, freqs)
    for t in (0, 1, 1023, 2047):
        assert torch.equal(y[t:t + 1], Q.rope(x[t:t + 1], pos[t:t + 1], freqs))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dt", sorted(DTYPES))
def test_strides_in_place_and_offsets(Q, dt, interleaved):
    """A view of a fused projection, in place, at an address that only the type aligns."""
    dtype = DTYPES[dt]
    T, H, D, r = 9, 4, 64, 32
    freqs, pos = Q.rope_frequencies(r)[0], _positions(T, 6).cuda()
    fused = _x(T, H + 2, D, dtype, 7).cuda()
    want = Q.rope(fused[:, 1:1 + H].contiguous(), pos, freqs, interleaved=interleaved)
    buf = fused.clone()
    view = buf[:, 1:1 + H]
    out = Q.rope(view, pos, freqs, interleaved=interleaved, out=view)
    assert out is view and torch.equal(view, want)
    assert torch.equal(buf[:, 0], fused[:, 0]) and torch.equal(buf[:, 1 + H:], fused[:, 1 + H:])
    odd = torch.empty(T * H * D + 1, dtype=dtype, device="cuda")[1:].view(T, H, D)
    odd.copy_(fused[:, 1:1 + H])
    assert torch.equal(Q.rope(odd, pos, freqs, interleaved=interleaved), want)
    heads_first = fused[:, 1:1 + H].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(Q.rope(heads_first, pos, freqs, interleaved=interleaved), want)


def test_gradient_is_the_transpose(Q):
    """<R x, g> = <x, R' g> term by term, and R' against differences of R (R is linear: one difference is exact up to
    rounding)."""
    T, H, D = 4, 2, 32
    x, g = _x(T, H, D, torch.float32, 8), _x(T, H, D, torch.float32, 9)
    pos, freqs = _positions(T, 10), Q.rope_frequencies(24, device="cpu")[0]
    dx = Q.rope(g.cuda(), pos.cuda(), freqs.cuda(), scale=1.5, backward=True).cpu().double()
    # every column of R from unit vectors
    num = torch.zeros(T, H, D, dtype=torch.float64)
    for d in range(D):
        e = torch.zeros_like(x)
        e[..., d] = 1.0
        col = Q.rope((x + e).cuda(), pos.cuda(), freqs.cuda(), scale=1.5).cpu().double() - \
            Q.rope(x.cuda(), pos.cuda(), freqs.cuda(), scale=1.5).cpu().double()
        num[..., d] = (col * g.double()).sum(-1)
    # each of the two values is within 7 * 2^-24 * 1.5 (|x1| + |x2| + 1) of R's (rope_bound with the fp32 rounding), in
    # all D of them times |g|
    tol = 2 * 1.5 * 7 * 2.0 ** -24 * (2 * x.abs().amax() + 1).item() * g.abs().double().sum(-1, keepdim=True)
    far = 2 * 3.2 * pos.double()[:, None, None] * 2.0 ** -53 * 2 * x.abs().amax().item() * g.abs().double().sum(-1, keepdim=True)
    assert bool(((dx - num).abs() <= tol + far).all())


def test_empty(Q):
    freqs = Q.rope_frequencies(64)[0]
    for T, H in ((0, 4), (3, 0)):
        y = Q.rope(torch.empty(T, H, 64, dtype=torch.float16, device="cuda"),
                   torch.zeros(T, dtype=torch.int64, device="cuda"), freqs)
        assert y.shape == (T, H, 64)


def test_refusals(Q):
    x = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    pos, freqs = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    with pytest.raises(ValueError):
        Q.rope(x, pos[:2], freqs)
    with pytest.raises(ValueError):
        Q.rope(x, pos.int(), freqs)
    with pytest.raises(ValueError):
        Q.rope(x, pos, freqs.float())
    with pytest.raises(ValueError):
        Q.rope(x.transpose(1, 2), pos, freqs)
    with pytest.raises(ValueError):
        Q.rope(x, pos, freqs, out=torch.empty(3, 2, 32, dtype=torch.float16, device="cuda"))
    with pytest.raises(Q.QuartzError):
        Q.rope(x, pos, torch.ones(64, dtype=torch.float64, device="cuda"))       # more than the head has
