"""Infinities and NaN in what is attended stay where quartz.h says: a query's in
its own row, a value's in its own element (encoded: its group of 64)."""
import pytest

import paged_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
PAGE, D, H, GROUP = 16, 128, 2, 4
PLANS = [[70, 33], [777], [2500, 0, 90]]  # one split or a cluster; a cluster; many splits


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _case(Q, store, lens, spoil=None):
    dtype = torch.bfloat16 if store == "bf16" else torch.float16
    width = -(-max(lens) // PAGE)
    table = torch.arange(width * len(lens), dtype=torch.int32).view(len(lens), width)
    kw = dict(params=Q.Params(group_s=16)) if store == "lzs" else dict(dtype=dtype)
    c = Q.empty_paged_cache(width * len(lens), PAGE, H, D, **kw)
    g = torch.Generator().manual_seed(sum(lens))
    k, v = (torch.randn(sum(lens), H, D, generator=g).to(dtype) for _ in range(2))
    if spoil is not None:
        t, value = spoil
        v[t, 1, 5] = value
    slots = torch.cat([table[b].long()[torch.arange(n) // PAGE] * PAGE + torch.arange(n) % PAGE for b, n in enumerate(lens)])
    Q.paged_append(c, k.cuda(), v.cuda(), slots.cuda())
    q = torch.randn(len(lens), H * GROUP, D, generator=g).to(dtype)
    return c, table, torch.tensor(lens, dtype=torch.int32), q


@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("lens", PLANS)
@pytest.mark.parametrize("token", [0, 17, -1])
def test_a_value(Q, store, value, lens, token):
    """Against the same call with a finite element: all others are the same bits."""
    t = token % lens[0]
    weights = [torch.zeros(len(lens), H, 16 * (-(-max(lens) // PAGE)), device="cuda") for _ in range(2)]
    out = []
    for x, w in zip((0.5, value), weights):
        c, table, ln, q = _case(Q, store, lens, (t, x))
        out.append(Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), D ** -0.5, weights=w))
        out.append(Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), D ** -0.5))
    assert Q.device_status() == 0 and torch.equal(*weights)
    hit = torch.zeros(len(lens), H * GROUP, D, dtype=torch.bool, device="cuda")
    hit[0, GROUP:, slice(0, 64) if store == "lzs" else 5] = True
    # what the page holds counts: the encoder leaves a NaN out of the group's maximum and stores a finite code for it
    held = R.held(c)[1][t // PAGE, t % PAGE, 1, 5].isfinite().item()
    assert held == (store == "lzs" and value != value)
    for good, bad in ((out[0], out[2]), (out[1], out[3])):
        assert torch.equal(good[~hit], bad[~hit]) and bool(good.isfinite().all())
        assert bool((bad[0, GROUP:, 5].isfinite() == held).all())


@pytest.mark.parametrize("store", ["f16", "bf16", "lzs"])
@pytest.mark.parametrize("lens", PLANS)
def test_a_query(Q, store, lens):
    """One head of NaN beside heads that share its tiles: those stay within the bound."""
    c, table, ln, q = _case(Q, store, lens)
    q[0, 2] = float("nan")
    o = Q.attention_paged(q.cuda(), c, table.cuda(), ln.cuda(), D ** -0.5, out_dtype=torch.float32).cpu()
    assert Q.device_status() == 0 and bool(o[0, 2].isnan().all())
    finite = q.clone()
    finite[0, 2] = 0
    k, v = R.held(c)
    ref, add, mag, pv = R.attention(finite, k, v, table, ln, D ** -0.5)
    bound, _ = R.attention_bounds(mag, pv, ref, add, max(lens), D, GROUP, torch.float32, 22 if store == "f16" else 17,
                                  float(v.nan_to_num(0, 0, 0).abs().max()))
    keep = torch.ones(len(lens), H * GROUP, dtype=torch.bool)
    keep[0, 2] = False
    assert bool(((o.double() - ref).abs() <= bound)[keep].all())
