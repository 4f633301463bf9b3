"""How far an angle may be off, by the stated bound: |position| (2^-63 f + 2^-64)
turns for a frequency of f turns per position, far below what a product in
binary64 (2^-53 f) would leave."""
import math

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


def _angle_bound(positions, freqs):
    """Radians [tokens, pairs]: the frequency's error times the position, and the last conversion to binary32, 2^-24 of at
    most an eighth of a turn."""
    turns = freqs.double().abs() / (2 * math.pi)
    far = positions.double().abs()[:, None] * (turns * 2.0 ** -63 + 2.0 ** -64)
    return 2 * math.pi * (far + 2.0 ** -24 / 8)


POSITIONS = [[0, 1, -1, 4095, 131071, 1 << 20, -(1 << 20) - 7], [1 << 31, (1 << 35) + 12345, -(1 << 35), (1 << 40) + 99991],
             [(1 << 45) + 3, -(1 << 47) - 1, (1 << 50) + 77777]]


@pytest.mark.parametrize("positions", POSITIONS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("scaling", ["none", "llama3", "odd"])
def test_angles_are_within_the_bound(Q, positions, interleaved, scaling):
    """Unit vectors: the result is the sine and the cosine themselves."""
    if scaling == "odd":  # frequencies past a turn per position, tiny, negative, zero, not normal
        freqs = torch.tensor([1e5, -0.3, 7.5, 1e-300, 5e-324, 0.0, 2.0 ** -60, math.pi], dtype=torch.float64)
    else:
        freqs, _ = Q.rope_frequencies(64, base=500000.0, scaling=scaling, factor=8.0 if scaling != "none" else 1.0, device="cpu")
    pos, n = torch.tensor(positions), len(freqs)
    i = torch.arange(n)
    i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    x = torch.zeros(len(positions), 1, 2 * n)
    x[..., i1] = 1.0
    y = Q.rope(x.cuda(), pos.cuda(), freqs.cuda(), interleaved=interleaved).cpu().double()
    a = R.angles(positions, freqs.tolist())
    # sine and cosine to an ulp of at most one (2^-24), the factor, the product and the sum half an ulp each
    tol = _angle_bound(pos, freqs) + 3 * 2.0 ** -24
    assert bool(((y[:, 0, i1] - a.cos()).abs() <= tol).all())
    assert bool(((y[:, 0, i2] - a.sin()).abs() <= tol).all())


def test_the_appended_keys_have_the_same_angles(Q):
    positions = POSITIONS[1]
    freqs = Q.rope_frequencies(64, base=500000.0)[0]
    k = torch.randn(len(positions), 2, 64, generator=torch.Generator().manual_seed(3)).half().cuda()
    pos, slots = torch.tensor(positions, device="cuda"), torch.arange(len(positions), device="cuda")
    c = Q.empty_paged_cache(1, 16, 2, 64, dtype=torch.float16)
    Q.paged_append(c, k, k, slots, positions=pos, freqs=freqs)
    assert Q.device_status() == 0 and torch.equal(c.k[0, :len(positions)], Q.rope(k, pos, freqs))
