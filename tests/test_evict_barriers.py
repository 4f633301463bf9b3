"""The choice's shared memory, read from the source: along every way through
the kernel (its loop with barriers skipped, run once, run twice) a barrier
lies between what one warp reads of a shared place and what another then
stores there, and the other way round.  Skipped is the way of equal weights:
all zero, all NaN, or one value."""
import pathlib
import re

import pytest

SOURCE = pathlib.Path(__file__).resolve().parents[1] / "paper_2509_26436_gb300" / "csrc" / "evict.cu"
BARRIER = "__syncthreads()"


def _block(text, start):
    """Text from the brace at or behind `start` to its partner, without them, and the place behind."""
    i = text.index("{", start)
    depth, j = 0, i
    while True:
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i + 1:j], j + 1
        j += 1


def _kernel():
    text = re.sub(r"//[^\n]*", "", SOURCE.read_text())
    return _block(text, text.index("evict_select_kernel(SelectArgs a)"))[0]


def _parts(body):
    """Before the first loop that holds a barrier, its body, behind it."""
    for m in re.finditer(r"\b(?:while|for) \([^{;]*(?:;[^{;]*;[^{;]*)?\) \{", body):
        loop, behind = _block(body, m.end() - 1)
        if BARRIER in loop:
            return body[:m.start()], loop, body[behind:]
    return body, "", ""


def _shared(body):
    names = []
    for decl in re.findall(r"__shared__ uint32_t ([^;]+);", body):
        names += [n.split("[")[0].strip() for n in decl.split(",")]
    return names


def _steps(code, names):
    """(barrier, None) and (read | write, array) in the order of the text, a statement at a time."""
    code = re.sub(r"(extern )?__shared__[^;]+;", "", code)
    for statement in re.split(r"[;{}]", code):
        if BARRIER in statement:
            yield "barrier", None
            continue
        if "auto key_at" in statement:
            continue
        reads, writes = [], []
        for name in names:
            place = re.escape(name) + r"\b(?:\[[^\[\]]*(?:\[[^\[\]]*\][^\[\]]*)*\])?"
            for m in re.finditer(place, statement):
                stored = re.match(r"\s*=[^=]", statement[m.end():]) or statement[:m.start()].endswith("atomicAdd(&")
                (writes if stored else reads).append(name)
        if "key_at(" in statement:
            reads.append("s_keys")
        yield from (("read", n) for n in reads)
        yield from (("write", n) for n in writes)


@pytest.mark.parametrize("trips", [0, 1, 2])
def test_a_barrier_between_reads_and_stores(trips):
    body = _kernel()
    names = _shared(body)
    before, loop, behind = _parts(body)
    last, seen = {}, set()
    for what, name in _steps(";".join([before] + [loop] * trips + [behind]), names):
        if what == "barrier":
            last.clear()
            continue
        seen.add((what, name))
        assert last.get(name, what) == what, f"{name}: a {what} behind a {last[name]} without a barrier"
        last[name] = what
    # the text was understood: every array is stored and read on the way through the loop
    if trips:
        assert names and all({("read", n), ("write", n)} <= seen for n in names), seen
