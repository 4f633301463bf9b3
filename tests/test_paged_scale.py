"""A softmax scale whose product with log2 e leaves binary32 is refused: q . k = 0
would meet an infinity in the kernels."""
import ctypes as C
import math

import pytest

from paper_2509_26436_gb300 import _native as N
from paper_2509_26436_gb300 import build as B

torch = pytest.importorskip("torch")
P = 0x10000  # an aligned address that no check dereferences
MOST = 2.3586e38  # below 2^128 (1 - 2^-24) / log2 e = 2.35866e38


def _call(scale):
    side = N.QuartzPages()
    side.data, side.stride_page, side.stride_slot, side.stride_head = P, 4096, 256, 128
    c = N.QuartzPagedCache(N.PAGES_F16, 16, 2, 128, 4, side, side)
    return N.load().quartz_paged_attention(P, 256, 128, 1, 2, C.byref(c), P, 4, P, 64, 0, scale, P, 0, None, 0, 0, P, 0, None)


def test_refused():
    B.build()
    for scale in (2.36e38, 3e38, -3e38, math.inf, math.nan):
        assert _call(scale) == N.QUARTZ_ERR_INVALID_ARG, scale
    for scale in (MOST, -MOST, 0.0):  # taken, up to the workspace
        assert _call(scale) == N.QUARTZ_ERR_WORKSPACE


@pytest.mark.gpu
def test_the_largest_scale():
    """Scores of 0 at the largest scale: every token weighs the same."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    n, D = 33, 64
    c = Q.empty_paged_cache(3, 16, 1, D, dtype=torch.float16)
    v = torch.ones(n, 1, D, dtype=torch.float16, device="cuda")
    Q.paged_append(c, v, v, torch.arange(n, device="cuda"))
    args = (torch.zeros(1, 1, D, dtype=torch.float16, device="cuda"), c, torch.arange(3, dtype=torch.int32, device="cuda")[None],
            torch.tensor([n], dtype=torch.int32, device="cuda"))
    assert bool((Q.attention_paged(*args, MOST) == 1.0).all()) and Q.device_status() == 0
    with pytest.raises(Q.QuartzError):
        Q.attention_paged(*args, 3e38)
