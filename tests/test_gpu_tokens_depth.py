"""Positions of drafted tokens whose masks leave their own bit out: a token's depth is
the number of other drafted tokens that it sees."""
import pytest

import tokens_reference as R
from test_gpu_tokens_attention import DTYPES, Case, _trees

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _places(n, m, tree):
    base = n - m
    pos = [base + sum(1 for i in range(m) if i != j and t >> i & 1) for j, t in enumerate(tree)]
    return torch.tensor(pos), torch.tensor(list(range(base)) + pos)


def _seen(n, m, tree, window, pos, place):
    out = torch.ones((m, n), dtype=torch.bool)
    out[:, n - m:] = torch.tensor([[t >> i & 1 == 1 for i in range(m)] for t in tree])
    return out & (place[None] > pos[:, None] - window) if window else out


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("window,sloped", [(0, True), (1, False), (3, False), (20, True)])
@pytest.mark.parametrize("own", ["none", "some"])
def test_masks_of_ancestors(Q, kind, window, sloped, own):
    """Ancestors alone (a verifier that adds a token's own key elsewhere), or some tokens' own bits as well."""
    seqs = [(140, 12), (64, 64), (300, 61), (9, 1)]
    tree, at = _trees(seqs, 3), 0
    for n, m in seqs:
        for j in range(m):
            if own == "none" or j % 3:
                tree[at + j] &= ~(1 << j)
        at += m
    slopes = 2.0 ** -torch.arange(1, 7, dtype=torch.float32) if sloped else None
    c = Case(Q, kind, 128, 2, 3, 16, seqs, seed=window)
    signed = torch.tensor([t - (1 << 64) if t >> 63 else t for t in tree]).cuda()
    o = Q.attention_paged_tokens(c.q.cuda(), c.cache, *c.args, 0.1, tree=signed, window=window,
                                 slopes=None if slopes is None else slopes.cuda(), out_dtype=torch.float32)
    for b, (n, m) in enumerate(seqs):
        s0 = c.starts[b]
        pos, place = _places(n, m, tree[s0:s0 + m])
        ref, bound = R.attention(c.q[s0:s0 + m], c.k[b], c.v[b], 0.1, _seen(n, m, tree[s0:s0 + m], window, pos, place),
                                 DTYPES[kind], pos, place, 0.0, slopes)
        off = (o[s0:s0 + m].cpu().double() - ref).abs() - R.rounded(bound, ref, o.dtype)
        assert bool((off <= 0).all()), (b, n, m, float(off.max()))
    assert Q.device_status() == 0
