"""Scores between -3e38 and the lowest binary32 number, -(2 - 2^-23) 2^127 =
-3.4028e38: finite, so that equal ones weigh the same, and a higher one beside
them takes all."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
D, PAGE = 64, 16


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _scale(target):
    """A scale that makes q . k = -2^30 a score of `target` in units of ln 2 (what is compared in the kernels)."""
    return -target * math.log(2) / 2.0 ** 30


@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
@pytest.mark.parametrize("target", [-3.05e38, -3.3e38, -3.4e38])
@pytest.mark.parametrize("lens,H", [([5, 900, 0, 1], 2), ([777], 40), ([3000] * 2, 8), ([9001], 1)])
def test_equal_scores_near_the_lowest_number(Q, store, target, lens, H):
    dtype = torch.bfloat16 if store == "bf16" else torch.float16
    width = -(-max(lens) // PAGE)
    pages = width * len(lens)
    c = Q.empty_paged_cache(pages, PAGE, H, D, **(dict(params=Q.Params(group_s=16)) if store == "lzs" else dict(dtype=dtype)))
    table = torch.arange(pages, dtype=torch.int32).view(len(lens), width)
    t = [torch.arange(n) for n in lens]
    slots = torch.cat([table[b].long()[i // PAGE] * PAGE + i % PAGE for b, i in enumerate(t)])
    # keys of one value per row: 127 x 2^5 (of 64 equal elements the group's scale is 2^5, the code 7 2^4 = 112)
    size = 4064.0 if store == "lzs" else 4096.0
    held = 3584.0 if store == "lzs" else 4096.0
    k = torch.full((len(slots), H, D), size, dtype=dtype)
    # values: one number per row and head, encoded to 112 / 127 of it exactly (the scale is a power of two)
    g = torch.Generator().manual_seed(1)
    exact = torch.randint(-3, 4, (len(slots), H, 1), generator=g).float()
    v = (127.0 * 2.0 ** exact).expand(-1, -1, D).to(dtype)
    if store == "bf16":
        v = (112.0 * 2.0 ** exact).expand(-1, -1, D).to(dtype)  # bf16 holds 8 bits
    Q.paged_append(c, k.cuda(), v.contiguous().cuda(), slots.cuda())
    vals = (112.0 if store != "f16" else 127.0) * 2.0 ** exact[..., 0].double()
    # q . k = 64 held q: -2^30 with 16-bit keys, with encoded ones -7/8 2^30
    q = torch.full((len(lens), H, D), -4096.0, dtype=dtype)
    scale = _scale(target) * 4096.0 / held
    assert math.isfinite(scale * 1.4427) and abs(scale * 64 * held * 4096 * 1.442695) < 3.4028e38
    w = torch.zeros(len(lens), H, width * PAGE, device="cuda")
    ln = torch.tensor(lens, dtype=torch.int32)
    args = (q.cuda(), c, table.cuda(), ln.cuda(), scale)
    a = Q.attention_paged(*args, out_dtype=torch.float32)
    b = Q.attention_paged(*args, out_dtype=torch.float32, weights=w)
    at = 0
    for i, n in enumerate(lens):
        mine = vals[at:at + n]
        at += n
        want = mine.mean(0) if n else torch.zeros(H, dtype=torch.float64)
        # weights of 2^0 are exact; n / 16 + 64 steps of 2^-23 in each of two sums and the division's 2^-23
        tol = want * (2 * (n / 16 + 64) + 1) * 2.0 ** -23
        for o in (a, b):
            assert bool(((o[i].cpu().double() - want[:, None]).abs() <= tol[:, None]).all())
        got = w[i, :, :n].cpu().double()
        assert bool(((got * n - 1).abs() <= (n / 16 + 72) * 2.0 ** -23).all()) and not w[i, :, n:].any()
    assert Q.device_status() == 0


@pytest.mark.parametrize("store", ["f16", "bf16"])
@pytest.mark.parametrize("place", [0, 333, 899])
def test_a_higher_score_takes_all(Q, store, place):
    """899 tokens at -3.3e38, one at half of that: the one's value."""
    dtype, n, H = (torch.bfloat16 if store == "bf16" else torch.float16), 900, 2
    width = -(-n // PAGE)
    c = Q.empty_paged_cache(width, PAGE, H, D, dtype=dtype)
    k = torch.full((n, H, D), 4096.0, dtype=dtype)
    k[place] = 2048.0
    v = torch.ones(n, H, D, dtype=dtype)
    v[place] = 5.0
    Q.paged_append(c, k.cuda(), v.cuda(), torch.arange(n, device="cuda"))
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None]
    o = Q.attention_paged(torch.full((1, H, D), -4096.0, dtype=dtype, device="cuda"), c, table,
                          torch.tensor([n], dtype=torch.int32, device="cuda"), _scale(-3.3e38))
    assert Q.device_status() == 0 and bool((o == 5.0).all())
