"""How many bits the softmax weights of attention_paged_tokens() enter the value
product with: two parts of the pages' type for few rows and for binary32 results."""
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


def _check(c, o, scale, tree=None, **shape):
    """Against 64 bits, with tokens_reference's bound for weights that are not rounded, and what two parts lose: each half a
    step, so eps^2 / 4 of a weight; and fp16, whose second parts end at 2^-24 (weights are 2^8 at the most when they are
    written, up to 2^7 more later), 2^-25 2^-8 of the largest weight for each token seen."""
    dtype = DTYPES[c.kind]
    half = torch.finfo(dtype).eps / 2
    for b, (n, m) in enumerate(c.seqs):
        s0 = c.starts[b]
        t = None if tree is None else tree[s0:s0 + m]
        pos, place = R.places(n, m, t)
        ref, bound = R.attention(c.q[s0:s0 + m], c.k[b], c.v[b], scale, R.seen(n, m, t), torch.float32, torch.tensor(pos),
                                 torch.tensor(place), shape.get("cap", 0.0), shape.get("slopes"))
        size = c.v[b].double().abs().repeat_interleave(c.G, 1)  # [token, q head, element]
        low = 2.0 ** -33 * size.sum(0) if dtype == torch.float16 else 0.0
        bound = bound + 1.01 * half ** 2 * size.amax(0, keepdim=True) + low
        off = (o[s0:s0 + m].cpu().double() - ref).abs() - R.rounded(bound, ref, o.dtype)
        assert bool((off <= 0).all()), (b, n, m, float(off.max()))


def _signed(tree):
    return None if tree is None else torch.tensor([t - (1 << 64) if t >> 63 else t for t in tree]).cuda()


# one token, a tree, sequences of which one has all 128 rows of a tile; long enough to be cut; short enough not to be
FEW = [[(1000, 1), (17, 1)], [(300, 61), (70, 5), (64, 64)], [(5000, 9)]]


@pytest.mark.parametrize("out", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("seqs", FEW)
def test_few_rows(Q, kind, D, out, seqs):
    c = Case(Q, kind, D, 2, 2, 16, seqs, seed=D)
    tree = _trees(seqs, 1)
    o = Q.attention_paged_tokens(c.q.cuda(), c.cache, *c.args, D ** -0.5, tree=_signed(tree), out_dtype=out, max_new=64)
    _check(c, o, D ** -0.5, tree)


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("shape", ["plain", "cap", "slopes"])
def test_binary32_results_of_many_rows(Q, kind, D, shape):
    seqs = [(300, 140), (1500, 33), (129, 129)]
    c = Case(Q, kind, D, 2, 3, 16, seqs, seed=D)
    how = {"plain": {}, "cap": dict(cap=5.0), "slopes": dict(slopes=2.0 ** -torch.arange(1, 7, dtype=torch.float32))}[shape]
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in how.items()}
    o = Q.attention_paged_tokens(c.q.cuda(), c.cache, *c.args, D ** -0.5, out_dtype=torch.float32, **dev)
    _check(c, o, D ** -0.5, **how)
