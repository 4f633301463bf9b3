"""The norm of each head and its gradient over the range that is allowed: heads whose
squares come near the ends of binary32."""
import pytest

import tokens_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


# eps = 0 needs a mean of the squares of 2^-126 (1.2e-38) or more
@pytest.mark.parametrize("size,eps", [(1e13, 1e-6), (1e14, 0.0), (1e15, 1e-6), (1e16, 0.0), (5e17, 1e-6), (1e-10, 0.0),
                                      (1e-13, 0.0), (1e-15, 0.0), (1e-17, 0.0), (1e-15, 1e-30)])
@pytest.mark.parametrize("dt", sorted(DTYPES))
@pytest.mark.parametrize("D,r", [(64, 64), (128, 0), (96, 64), (37, 6)])
def test_large_and_small_heads(Q, D, r, dt, size, eps):
    T, H, dtype = 5, 3, DTYPES[dt]
    g = torch.Generator().manual_seed(D)
    x, dy = ((torch.randn((T, H, D), generator=g) * s).to(dtype) for s in (size, 1.0))
    w = 1 + 0.2 * torch.randn(D, generator=g)
    freqs = pos = None
    if r:
        freqs, pos = 10000.0 ** (-torch.arange(r // 2, dtype=torch.float64) / (r // 2)), torch.randint(0, 1000, (T,), generator=g)
    dev = [None if t is None else t.cuda() for t in (x, w, dy, pos, freqs)]
    y, _ = Q.qk_norm_rope(dev[0], None, dev[1], None, *dev[3:], eps=eps)
    ref, bound = R.norm(x, w, eps, pos, freqs, None, False, 1.0)
    assert bool(((y.cpu().double() - ref).abs() <= R.rounded(bound, ref, dtype)).all())
    dx, _, dw, _ = Q.qk_norm_rope_backward(dev[2], None, dev[0], None, dev[1], None, *dev[3:], eps=eps)
    dx_ref, dw_ref, e_dx, e_dw = R.norm_grad(x, w, dy, eps, pos, freqs, None, False, 1.0)
    assert bool(((dx.cpu().double() - dx_ref).abs() <= R.rounded(e_dx, dx_ref, dtype)).all())
    assert bool(((dw.cpu().double() - dw_ref).abs() <= R.rounded(e_dw, dw_ref, torch.float32)).all())
    assert Q.device_status() == 0
