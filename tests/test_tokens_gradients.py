"""Gradients that would be lost are refused by every call for several new tokens."""
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def Q():
    from paper_2509_26436_gb300 import build as B
    B.build()
    import paper_2509_26436_gb300 as Q
    from paper_2509_26436_gb300 import paged
    if paged.torch is None:
        paged._bind()
    return Q


def _norm_args():
    return dict(dyq=torch.zeros(3, 2, 64), dyk=torch.zeros(3, 1, 64), q=torch.zeros(3, 2, 64), k=torch.zeros(3, 1, 64),
                wq=torch.ones(64), wk=torch.ones(64))


@pytest.mark.parametrize("name", ["dyq", "dyk", "q", "k", "wq", "wk"])
def test_second_derivatives(Q, name):
    """The gradient depends on all that it gets: under create_graph each may require one, with a constant dy as well."""
    t = _norm_args()
    t[name].requires_grad_(True)
    with pytest.raises(ValueError, match="records no gradient"):
        Q.qk_norm_rope_backward(*t.values())
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):  # the next check
        Q.qk_norm_rope_backward(*t.values())


def test_learned_frequencies(Q):
    freqs = torch.ones(32, dtype=torch.float64, requires_grad=True)
    pos, axis = torch.zeros(3, dtype=torch.int64), torch.zeros(32, dtype=torch.int32)
    t = _norm_args()
    for call in (lambda: Q.rope_axes(t["q"], pos[None], freqs, axis),
                 lambda: Q.qk_norm_rope(t["q"], t["k"], t["wq"], t["wk"], pos, freqs),
                 lambda: Q.qk_norm_rope_backward(*t.values(), pos, freqs)):
        with pytest.raises(ValueError, match="records no gradient"):
            call()


@pytest.mark.parametrize("name", ["q", "slopes", "out", "pool"])
def test_attention(Q, name):
    t = dict(q=torch.zeros(3, 2, 64), slopes=torch.ones(2), out=torch.zeros(3, 2, 64), pool=torch.zeros(4, 16, 1, 64))
    t[name].requires_grad_(True)
    cache = types.SimpleNamespace(_pools=(t["pool"], t["pool"]))
    lens, table = torch.tensor([3], dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError, match="records no gradient"):
        Q.attention_paged_tokens(t["q"], cache, table, lens, torch.tensor([0, 3], dtype=torch.int32), 0.125,
                                 slopes=t["slopes"], out=t["out"])


@pytest.mark.gpu
def test_on_the_device(Q):
    """The real calls: a second derivative in an autograd function, and attention with and without gradients."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, w):
            ctx.save_for_backward(q, w)
            return Q.qk_norm_rope(q, None, w, None)[0]

        @staticmethod
        def backward(ctx, g):
            # (a sum's gradient is broadcast, which is refused as any last dimension that is not contiguous)
            dq, _, dw, _ = Q.qk_norm_rope_backward(g.contiguous(), None, ctx.saved_tensors[0], None, ctx.saved_tensors[1], None)
            return dq, dw

    q, w = torch.randn(5, 2, 64, device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="records no gradient"):
        torch.autograd.grad(Norm.apply(q, w).sum(), (q, w), create_graph=True)
    assert all(g.isfinite().all() for g in torch.autograd.grad(Norm.apply(q, w).sum(), (q, w)))

    pools = [torch.randn(4, 16, 2, 64, device="cuda").half() for _ in range(2)]
    cache = Q.PagedCache(*pools, 16)
    args = (torch.arange(4, device="cuda").int()[None], torch.tensor([40], device="cuda").int(),
            torch.tensor([0, 5], device="cuda").int(), 0.125)
    x = q.detach().half().requires_grad_(True)
    with pytest.raises(ValueError, match="records no gradient"):
        Q.attention_paged_tokens(x, cache, *args)
    with torch.no_grad():
        want = Q.attention_paged_tokens(x, cache, *args)
    assert torch.equal(want, Q.attention_paged_tokens(x.detach(), cache, *args))
    pools[1].requires_grad_(True)
    with pytest.raises(ValueError, match="records no gradient"):
        Q.attention_paged_tokens(x.detach(), cache, *args)
