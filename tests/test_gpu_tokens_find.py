"""The cut of attention_paged_tokens() into runs of tiles, up to the largest sequences:
the kernel's own search, without the attention, against the same sums in Python."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2509_26436_gb300 import build as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
CTAS, KEYS, EDGE = 152, 128, 3


@pytest.fixture(scope="module")
def find(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    so = str(tmp_path_factory.mktemp("find") / "find.so")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "tokens_find.cu")
    subprocess.run([B.nvcc(), *B.ARCH, "-O2", "-std=c++17", "--expt-relaxed-constexpr", "-diag-suppress", "177", "-Xcompiler",
                    "-fPIC", "-I", B.INCLUDE, "-I", B.CSRC, "-shared", "-cudart", "shared", "-o", so, src], check=True)
    lib = C.CDLL(so)
    lib.find.argtypes = [C.c_int, C.c_void_p, C.c_void_p] + [C.c_int] * 7 + [C.c_void_p, C.c_void_p]
    return lib.find


def _tiles(n, m, group, rows):
    """Tiles of keys of each block of rows: causal, so up to the last row's position."""
    block = torch.arange(-(-m * group // rows), dtype=torch.int64)
    last = torch.minimum(torch.tensor(m - 1), (block * rows + rows - 1) // group)
    return (n - m + last) // KEYS + 1


# (rows of a CTA, heads, group, [(cached, new)]): a few short ones; one key head's tiles just below, above and far above 2^31
# and 2^32; several sequences that pass it together; behind others with little or nothing new
M = 1 << 20
CASES = [(256, 2, 3, [(300, 140), (5, 0), (1000, 257), (64, 1)]),
         (256, 1, 128, [(M - 4096, M - 4096)]), (256, 1, 128, [(M, M)]), (128, 1, 64, [(M + 77, M + 77)]),
         (128, 2, 128, [(M, M)]), (256, 3, 8, [(4 * M + 12345, 4 * M + 12345)]),
         (256, 2, 16, [(100, 3), (3 * M, 3 * M), (5, 0), (3 * M + 1, 2 * M), (900, 900)])]


@pytest.mark.parametrize("rows,heads,group,seqs", CASES)
def test_runs_are_equal_and_begin_where_the_last_ends(find, rows, heads, group, seqs):
    starts = [0]
    for _, m in seqs:
        starts.append(starts[-1] + m)
    lens = torch.tensor([n for n, _ in seqs], dtype=torch.int32).cuda()
    at = torch.tensor(starts, dtype=torch.int32).cuda()
    out, err = torch.zeros((CTAS, 8), dtype=torch.int64).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    assert find(rows, lens.data_ptr(), at.data_ptr(), len(seqs), starts[-1], max(n for n, _ in seqs),
                max(m for _, m in seqs), heads, group, CTAS, out.data_ptr(), err.data_ptr()) == 0
    assert err.item() == 0
    per = [_tiles(n, m, group, rows) for n, m in seqs]
    total = heads * sum(int(t.sum()) for t in per)
    edge = min(EDGE, total // (4 * CTAS))
    ends = [torch.cumsum(t + edge, 0) for t in per]  # of a key head's blocks
    sizes = [int(e[-1]) if len(e) else 0 for e in ends]
    everything = heads * sum(sizes)
    chunk = -(-everything // CTAS)
    for cta, (some, pos, end, got_edge, b, head, block, off) in enumerate(out.tolist()):
        want = chunk * cta
        assert got_edge == edge and pos == want and end == min(want + chunk, everything) and bool(some) == (want < everything)
        if not some:
            continue
        seq = 0
        while want >= heads * sizes[seq]:
            want -= heads * sizes[seq]
            seq += 1
        h, rest = divmod(want, sizes[seq])
        blk = int(torch.searchsorted(ends[seq], rest, right=True))
        assert (b, head, block, off) == (seq, h, blk, rest - (int(ends[seq][blk - 1]) if blk else 0))
