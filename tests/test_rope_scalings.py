"""rope_frequencies' long-context scalings, every pair, from what they mean: how
many turns a pair makes over the original length."""
import math

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def Q():
    from paper_2509_26436_gb300 import build
    build.build()
    import paper_2509_26436_gb300 as Q
    return Q


def _turns(i, rotary, base, length):
    return length * base ** (-2.0 * i / rotary) / (2 * math.pi)


# (rotary, base, original length, factor, beta_fast, beta_slow): ends inside the pairs, before the first, past the last
YARN = [(64, 500000.0, 8192, 8.0, 32.0, 1.0), (128, 10000.0, 4096, 16.0, 32.0, 1.0), (128, 1e6, 32768, 4.0, 32.0, 1.0),
        (16, 10000.0, 4096, 40.0, 32.0, 1.0), (64, 10000.0, 128, 4.0, 32.0, 1.0), (64, 10000.0, 1 << 20, 4.0, 32.0, 1.0),
        (64, 10000.0, 4096, 2.0, 4.0, 3.9), (96, 150000.0, 4096, 32.0, 8.0, 2.0), (2, 10000.0, 4096, 8.0, 32.0, 1.0)]


@pytest.mark.parametrize("rotary,base,length,factor,fast,slow", YARN)
def test_yarn(Q, rotary, base, length, factor, fast, slow):
    """Pairs up to the last that makes `fast` turns keep their frequency, those from the first that makes no more than
    `slow` have it divided; between, a straight line over the pairs' numbers.  Pairs are counted past both ends of the
    head, but the line starts no earlier than pair 0 and ends no later than pair rotary - 1."""
    far = range(-4 * rotary, 4 * rotary)
    lo = max(0, max(i for i in far if _turns(i, rotary, base, length) >= fast))
    hi = min(rotary - 1, min(i for i in far if _turns(i, rotary, base, length) <= slow))
    f, m = Q.rope_frequencies(rotary, base=base, scaling="yarn", factor=factor, original_length=length, beta_fast=fast,
                              beta_slow=slow, device="cpu")
    assert f.shape == (rotary // 2,) and m == pytest.approx(0.1 * math.log(factor) + 1, rel=1e-15)
    for i, got in enumerate(f.tolist()):
        plain = base ** (-2.0 * i / rotary)
        part = 0.0 if i <= lo else 1.0 if i >= hi else (i - lo) / (hi - lo)
        assert got == pytest.approx(plain * (1 - part) + plain / factor * part, rel=1e-14), i


@pytest.mark.parametrize("rotary,base,length,factor,low,high", [(64, 500000.0, 8192, 8.0, 1.0, 4.0), (128, 500000.0, 8192, 32.0, 1.0, 4.0),
                                                                (32, 10000.0, 2048, 4.0, 2.0, 9.0), (2, 10000.0, 1, 8.0, 1.0, 4.0)])
def test_llama3(Q, rotary, base, length, factor, low, high):
    """Over `high` turns as they are, under `low` divided, between in proportion to the turns."""
    f, m = Q.rope_frequencies(rotary, base=base, scaling="llama3", factor=factor, original_length=length, low_freq_factor=low,
                              high_freq_factor=high, device="cpu")
    assert m == 1.0
    for i, got in enumerate(f.tolist()):
        plain, turns = base ** (-2.0 * i / rotary), _turns(i, rotary, base, length)
        want = plain if turns >= high else plain / factor if turns <= low else \
            plain / factor + (plain - plain / factor) * (turns - low) / (high - low)
        assert got == pytest.approx(want, rel=1e-13), i


def test_a_factor_of_one_changes_nothing(Q):
    plain, _ = Q.rope_frequencies(64, device="cpu")
    for scaling in ("linear", "yarn", "llama3"):
        f, m = Q.rope_frequencies(64, scaling=scaling, factor=1.0, device="cpu")
        assert m == 1.0 and torch.allclose(f, plain, rtol=1e-15, atol=0)
