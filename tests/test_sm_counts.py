"""Plans ask the device for its number of SMs: the full chip's is written out in
one place, for sizes that are asked on a host without a device."""
import pathlib
import re

CSRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2509_26436_gb300" / "csrc"
MULTIPLES = {str(152 * n) for n in range(1, 17)}


def test_no_sm_count_is_written_out():
    found = []
    for path in sorted([*CSRC.glob("*.cu"), *CSRC.glob("*.cuh"), *CSRC.glob("*.h")]):
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", path.read_text(), flags=re.S)
        found += [(path.name, n) for n in re.findall(r"(?<![\w.])\d+(?![\w.])", code) if n in MULTIPLES]
    assert found == [("quartz_internal.h", "152")]
