"""New lengths written over the old ones while other heads read those: refused."""
import pytest

from paper_2509_26436_gb300 import _native as N
from paper_2509_26436_gb300 import build as B

torch = pytest.importorskip("torch")
P = 0x10000  # an aligned address that no check dereferences


@pytest.mark.parametrize("at", [0, 4, -4, 8, -8])
def test_overlapping_lengths_are_refused(at):
    B.build()
    assert N.load().quartz_evict_select(P, 64, 32, P, 3, 2, 32, 8, 2, 1, 2 * P, P + at, None) == N.QUARTZ_ERR_INVALID_ARG


@pytest.mark.gpu
def test_lengths_side_by_side():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    w = torch.rand(3, 2, 40, device="cuda")
    both = torch.tensor([7, 40, 8, -1, -1, -1], dtype=torch.int32, device="cuda")
    _, new = Q.evict_select(w, both[:3], 8, new_lens=both[3:])
    assert Q.device_status() == 0 and both.tolist() == [7, 40, 8, 7, 8, 8]
    with pytest.raises(Q.QuartzError):
        Q.evict_select(w, both[:3], 8, new_lens=both[:3])
    with pytest.raises(Q.QuartzError):
        Q.evict_select(w, both[1:4], 8, new_lens=both[3:])
