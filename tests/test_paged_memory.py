"""Where results get their memory: torch's short way to it is used only as long as it is
what it was, and not where torch fills new memory."""
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def paged():
    from paper_2509_26436_gb300 import build as B
    B.build()
    from paper_2509_26436_gb300 import paged
    if paged.torch is None:
        paged._bind()
    return paged


def _torch(f):
    guards = types.SimpleNamespace() if f is None else types.SimpleNamespace(_empty_strided_cuda=f)
    return types.SimpleNamespace(_C=types.SimpleNamespace(_dynamo=types.SimpleNamespace(guards=guards)), float16=torch.float16)


def _made(shape, stride, dtype):
    return types.SimpleNamespace(shape=shape, stride=lambda: stride, dtype=dtype, get_device=lambda: 0)


@pytest.mark.parametrize("f", [None, lambda shape, stride: None, lambda shape, stride, dtype: None,
                               lambda shape, stride, dtype: _made(shape, (4, 2, 1), dtype),
                               lambda shape, stride, dtype: _made(shape, stride, torch.float32)])
def test_another_version_of_it_is_not_used(paged, monkeypatch, f):
    monkeypatch.setattr(paged, "_device", lambda: 0)
    assert paged._quick_empty(_torch(f)) is None
    assert paged._quick_empty(_torch(_made)) is _made


def test_memory_that_torch_fills(paged, monkeypatch):
    def fail(*_):
        raise AssertionError

    monkeypatch.setattr(paged, "_empty_strided", fail)
    monkeypatch.setattr(torch, "are_deterministic_algorithms_enabled", lambda: True)
    assert paged._empty((2, 3, 4), torch.float16, "cpu", None).shape == (2, 3, 4)
    monkeypatch.setattr(torch, "are_deterministic_algorithms_enabled", lambda: False)
    with pytest.raises(AssertionError):
        paged._empty((2, 3, 4), torch.float16, "cpu", None)


@pytest.mark.gpu
@pytest.mark.parametrize("deterministic", [False, True])
def test_on_the_device(paged, deterministic):
    import paper_2509_26436_gb300 as Q
    x = torch.randn(5, 2, 64, device="cuda")
    want = Q.qk_norm_rope(x, None, None, None)[0]
    torch.use_deterministic_algorithms(deterministic)
    try:
        assert torch.equal(Q.qk_norm_rope(x, None, None, None)[0], want)
        assert bool(paged._empty((1000,), torch.float32, "cuda", None).isnan().all()) or not deterministic
    finally:
        torch.use_deterministic_algorithms(False)
