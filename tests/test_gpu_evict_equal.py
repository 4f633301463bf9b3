"""The choice where all weights between sinks and recent tokens are one value:
sums that are still zero, a constant, infinities, NaN.  The lowest indices stay."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _want(lens, heads, budget, recent, sinks):
    kept = torch.full((len(lens), heads, budget), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        if n <= budget:
            kept[b, :, :n] = torch.arange(n, dtype=torch.int32)
        else:  # the sinks and the first of those between are consecutive
            kept[b] = torch.cat([torch.arange(budget - recent), torch.arange(n - recent, n)]).int()
    return kept


# (lens, heads, budget, recent, sinks): more than 152 heads (short: small CTAs), few, more keys than a CTA holds; runs of
# tokens that leave most warps without any
SHAPES = [([40, 9, 8, 0, 1, 300, 8192] * 4, 8, 8, 2, 1), ([40, 33, 100], 3, 32, 4, 2), ([8193, 5000], 2, 4096, 100, 4),
          ([8200, 64] * 10, 16, 60, 0, 0), ([48 * 1024 + 5, 70], 2, 64, 32, 0), ([50] * 200, 1, 49, 30, 19)]


@pytest.mark.parametrize("value", [0.0, 0.25, float("nan"), float("inf"), -float("inf"), -0.0])
@pytest.mark.parametrize("lens,heads,budget,recent,sinks", SHAPES)
def test_equal_weights(Q, value, lens, heads, budget, recent, sinks):
    w = torch.full((len(lens), heads, max(lens)), value, device="cuda")
    ln = torch.tensor(lens, dtype=torch.int32)
    want = _want(lens, heads, budget, recent, sinks)
    for _ in range(20):  # back to back: CTAs of one call beside those of the next
        kept, new = Q.evict_select(w, ln.cuda(), budget, recent=recent, sinks=sinks)
    assert Q.device_status() == 0
    assert torch.equal(kept.cpu(), want) and torch.equal(new.cpu(), ln.clamp(max=budget))
