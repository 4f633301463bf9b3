"""The weights' gradients over many tokens: no row is lost between blocks, groups, CTAs
and the last sum.  The bound is below what one token adds, which is shown."""
import pytest

import tokens_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    return Q


def _additions(T, heads, sms):
    """Additions that a row goes through, at most.  A group of 4 to 32 lanes has every (groups / here)-th head of a token of
    each of its CTA's blocks of `here` tokens; a side has a third of the SMs at least (of CTAs: as many or twice as many);
    then up to 64 groups, every 32nd of up to 2 sms + 2 CTAs, and 32 warps."""
    most = 0
    for groups in (8, 16, 32, 64):
        for here in (1, 2, 4, 8, 16):
            if here <= groups:
                turns = -(-T // here) // (sms // 3) + 1
                most = max(most, turns * -(-heads // (groups // here)))
    return most + 64 + (2 * sms + 2) // 32 + 1 + 32


# (tokens, q heads, k heads, dim, rotary): blocks that do not divide the tokens, a single token behind whole blocks
SIZES = [(4099, 6, 2, 128, 128), (4097, 5, 3, 64, 64), (1999, 2, 2, 96, 64), (2049, 3, 2, 80, 0), (1025, 2, 1, 37, 6)]


@pytest.mark.parametrize("T,Hq,Hk,D,r", SIZES)
@pytest.mark.parametrize("dt", sorted(DTYPES))
def test_every_row_counts(Q, T, Hq, Hk, D, r, dt):
    dtype, g = DTYPES[dt], torch.Generator().manual_seed(T)
    q, k, gq, gk = (torch.randn((T, h, D), generator=g).to(dtype) for h in (Hq, Hk, Hq, Hk))
    wq, wk = (1 + 0.2 * torch.randn(D, generator=g) for _ in range(2))
    pos = freqs = None
    if r:
        pos, freqs = torch.randint(0, 9000, (T,), generator=g), 10000.0 ** (-torch.arange(r // 2, dtype=torch.float64) / (r // 2))
    dev = [None if t is None else t.cuda() for t in (gq, gk, q, k, wq, wk, pos, freqs)]
    got = Q.qk_norm_rope_backward(*dev)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for x, dy, w, dw in ((q, gq, wq, got[2]), (k, gk, wk, got[3])):
        ref = R.norm_grad(x, w, dy, 1e-6, pos, freqs, None, False, 1.0)[1]
        # norm_grad's bound with the sum's depth for the number of rows
        xd, H = x.double(), x.shape[1]
        rr = (xd.square().mean(-1, keepdim=True) + 1e-6) ** -0.5
        turned = R._turn(dy.double(), pos, freqs, None, False, 1.0, True)
        e_g = R.turn_bound(dy.double().abs(), 0.0, pos, freqs, None, False, 1.0)
        terms, n = turned * xd * rr, (xd * rr).abs()
        bound = (n * e_g + terms.abs() * (((D + 4) / 2 + 4 + 3 + _additions(T, H, sms)) * R.U)).sum((0, 1))
        assert bool(((dw.cpu().double() - ref).abs() <= R.rounded(bound, ref, torch.float32)).all())
        # each token, left out, would be seen
        one = terms.sum(1)  # [token, element]
        assert bool(((one.abs() > 2 * R.rounded(bound, ref, torch.float32)).any(-1)).all())
