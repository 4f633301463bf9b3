"""The choice of more heads than there are SMs, against a sort: the instance
of small CTAs (up to 8192 tokens) and the one past it, to both sides."""
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


def _weights(B, H, n, kind):
    g = torch.Generator().manual_seed(B * 1000 + n)
    if kind == "ties":
        return torch.randint(0, 3, (B, H, n), generator=g).float()
    if kind == "equal":
        return torch.full((B, H, n), 0.25)
    if kind == "odd":
        special = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 1.0, -1.0, 3e38])
        return special[torch.randint(0, len(special), (B, H, n), generator=g)]
    return torch.exp(1.5 * torch.randn(B, H, n, generator=g))


@pytest.mark.parametrize("kind", ["sums", "ties", "odd", "equal"])
@pytest.mark.parametrize("n", [8192, 8193])
@pytest.mark.parametrize("budget,recent,sinks", [(256, 32, 4), (700, 0, 0), (1, 0, 0), (255, 250, 5)])
def test_more_heads_than_sms(Q, n, kind, budget, recent, sinks):
    """20 x 8 heads: empty, one token, at the budget and around it, up to the whole width."""
    around = [0, 1, budget - 1, budget, budget + 1, budget + 2, 2 * budget + 31]
    lens = around + [n, n - 1, 4097, 2048, 2047, 31, 33, 1000, 257, 511, 64, 100, 777]
    w, ln = _weights(len(lens), 8, n, kind), torch.tensor(lens, dtype=torch.int32)
    kept, new = Q.evict_select(w.cuda(), ln.cuda(), budget, recent=recent, sinks=sinks)
    assert Q.device_status() == 0
    want, want_new = R.evict(w, ln, budget, recent, sinks)
    assert torch.equal(new.cpu(), want_new) and torch.equal(kept.cpu(), want)


@pytest.mark.parametrize("B,H", [(152, 1), (153, 1), (19, 8), (9, 17)])
def test_around_the_number_of_sms(Q, B, H):
    """Heads on both sides of where the CTAs become small; strided weights and a stated bound."""
    n = 900
    w = _weights(B, H + 2, n + 3, "sums")
    ln = torch.tensor([(i * 211) % (n + 1) for i in range(B)], dtype=torch.int32)
    kept, _ = Q.evict_select(w.cuda()[:, 1:1 + H], ln.cuda(), 100, recent=7, sinks=2, max_len=n)
    want, _ = R.evict(w[:, 1:1 + H], ln, 100, 7, 2)
    assert Q.device_status() == 0 and torch.equal(kept.cpu(), want)


def test_a_bad_length_is_reported(Q):
    w = _weights(160, 1, 64, "sums").cuda()
    for bad in (65, -3):
        ln = torch.full((160,), 20, dtype=torch.int32)
        ln[77] = bad
        kept, _ = Q.evict_select(w, ln.cuda(), 8)
        assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX
        want, _ = R.evict(w.cpu(), torch.full((160,), 20, dtype=torch.int32), 8, 0, 0)
        others = [i for i in range(160) if i != 77]
        assert torch.equal(kept.cpu()[others], want[others])
