"""rope() loses no gradient without a word: where autograd would expect one it
refuses, and inside an autograd function both directions are the kernel's."""
import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("which", ["x", "out"])
def test_a_gradient_that_would_be_lost_is_refused(which):
    import paper_2509_26436_gb300 as Q
    from paper_2509_26436_gb300 import build
    build.build()
    x, out = torch.zeros(3, 2, 64), torch.zeros(3, 2, 64)
    (x if which == "x" else out).requires_grad_(True)
    args = (x, torch.zeros(3, dtype=torch.int64), torch.ones(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="records no gradient"):
        Q.rope(*args, out=out if which == "out" else None)
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):  # past that check: this is a tensor of the host
        Q.rope(*args, out=out if which == "out" else None)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_as_an_autograd_function(interleaved):
    """The documented way: gradients of an upstream weight against those of the rotation as a matrix of unit vectors."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    T, H, D = 5, 2, 16
    freqs, pos = Q.rope_frequencies(12)[0], torch.arange(T, device="cuda") * 7

    class Rope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return Q.rope(x, pos, freqs, interleaved=interleaved)

        @staticmethod
        def backward(ctx, g):
            return Q.rope(g.contiguous(), pos, freqs, interleaved=interleaved, backward=True)

    gen = torch.Generator().manual_seed(1)
    x = torch.randn(T, H, D, generator=gen).cuda().requires_grad_(True)
    g = torch.randn(T, H, D, generator=gen).cuda()
    with pytest.raises(ValueError):
        Q.rope(x, pos, freqs)
    Rope.apply(x).backward(g)
    with torch.no_grad():
        assert Q.rope(x, pos, freqs, interleaved=interleaved).requires_grad is False
    unit = torch.eye(D, device="cuda")[:, None, None].expand(D, T, H, D).contiguous()
    want = torch.stack([(Q.rope(u, pos, freqs, interleaved=interleaved).double() * g.double()).sum(-1) for u in unit], -1)
    # each column's two entries are cosine and sine to 5 * 2^-24; the gradient's two products and sum likewise
    tol = 16 * 2.0 ** -24 * g.abs().double().sum(-1, keepdim=True)
    assert bool(((x.grad.double() - want).abs() <= tol).all())
