"""The device error word keeps both kinds of error, and a timeout is told first."""
import os
import pathlib
import re
import subprocess

import pytest

torch = pytest.importorskip("torch")
ROOT = pathlib.Path(__file__).resolve().parents[1]
CSRC = ROOT / "paper_2509_26436_gb300" / "csrc"


def test_status_of_every_word(tmp_path):
    """0 none, 1 timeout, 2 index, 3 both."""
    src = tmp_path / "word.cpp"
    src.write_text("""#include "quartz_internal.h"
using namespace quartz;
static_assert(device_word_status(0) == QUARTZ_OK, "");
static_assert(device_word_status(QUARTZ_DEV_TIMEOUT) == QUARTZ_ERR_TIMEOUT, "");
static_assert(device_word_status(QUARTZ_DEV_INDEX) == QUARTZ_ERR_INDEX, "");
static_assert((QUARTZ_DEV_TIMEOUT | QUARTZ_DEV_INDEX) == 3 && device_word_status(3) == QUARTZ_ERR_TIMEOUT, "");
""")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++17", "-fsyntax-only", f"-I{ROOT / 'include'}", f"-I{CSRC}", f"-I{cuda}/include", str(src)],
                   check=True)


def test_kernels_only_add_to_the_word():
    """No kernel stores over what another one recorded."""
    found = 0
    for path in sorted([*CSRC.glob("*.cu"), *CSRC.glob("*.cuh")]):
        code = re.sub(r"//[^\n]*", "", path.read_text())
        for m in re.finditer(r"atomic(\w+)\(\s*[\w.]*dev_err\b", code):
            assert m.group(1) == "Or", f"{path.name}: atomic{m.group(1)} on the error word"
            found += 1
        assert not re.search(r"(?<!int )\*[\w.]*dev_err\s*=[^=]", code), path.name
    assert found >= 8


@pytest.mark.gpu
@pytest.mark.parametrize("index_first", [False, True])
def test_an_index_does_not_hide_a_timeout(index_first):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2509_26436_gb300 as Q
    w, ln = torch.rand(1, 1, 16, device="cuda"), torch.tensor([17], dtype=torch.int32, device="cuda")
    assert Q.device_status() == 0
    if index_first:
        Q.evict_select(w, ln, 4)
    Q.selftest_timeout(1_000_000)
    if not index_first:
        Q.evict_select(w, ln, 4)
    assert Q.device_status() == Q._native.QUARTZ_ERR_TIMEOUT and Q.device_status() == 0
    Q.evict_select(w, ln, 4)
    assert Q.device_status() == Q._native.QUARTZ_ERR_INDEX and Q.device_status() == 0
