"""Which calls of attention of several new tokens keep their blocks whole (their
workspace is the 256 bytes that nothing is written to), and that results are right on
both sides of the borders."""
import ctypes as C

import pytest

from paper_2509_26436_gb300 import _native as N
from test_paged_abi import _cache
from test_tokens_abi import lib  # noqa: F401

torch = pytest.importorskip("torch")
F16, LZS = N.PAGES_F16, N.PAGES_ENCODED


# (pages, dim, blocks): most keys that stay whole; 152 SMs, 8 new tokens a sequence
@pytest.mark.parametrize("kind,dim,blocks,keys", [(F16, 64, 1, 1024), (F16, 128, 40, 1024), (F16, 128, 152, 1024),
                                                  (F16, 192, 1, 512), (F16, 256, 76, 512), (F16, 256, 80, 1024),
                                                  (LZS, 128, 1, 512), (LZS, 64, 76, 512), (LZS, 128, 80, 1024),
                                                  (F16, 128, 160, 0), (LZS, 256, 160, 0)])
def test_where_blocks_stay_whole(lib, kind, dim, blocks, keys):  # noqa: F811
    if torch.cuda.is_available() and torch.cuda.get_device_properties(0).multi_processor_count != 152:
        pytest.skip("another number of SMs")
    heads = blocks if blocks < 100 else blocks // 4
    seqs = blocks // heads
    c = _cache(kind, heads=heads, dim=dim, pages=100, page=128)
    for n in (256, 512, 513, 1024, 1025, 4096):
        # one new token a sequence: a block for each key head of it, and none of 128 rows to fill
        size = lib.quartz_paged_attention_tokens_workspace_size(C.byref(c), seqs, seqs, heads, n, 1)
        assert (size == 256) == (n <= keys), n


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "lzs"])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("n", [511, 512, 513, 1024, 1025])
def test_results_around_the_borders(kind, D, n):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    from test_gpu_tokens_attention import Case, _trees
    for seqs in ([(n, 8)], [(n, 3), (n - 100, 8), (7, 7), (n - 1, 1)] * 5):
        c = Case(Q, kind, D, 4, 2, 16, seqs, seed=n)
        # bounds that hold exactly, so that the table's width does not decide
        c.run(Q, max_len=n, max_new=8, tree=_trees(seqs, n))
