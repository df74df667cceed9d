"""Rules that the kernels' source has to keep and that no run can show: a missing fence does not fail, it only may (CPU only)."""
import glob
import os
import re

import pytest

from paper_2506_12355_b200 import build

SOURCES = sorted(glob.glob(os.path.join(build.CSRC, "*.cuh")))


def without_comments(text):
    return re.sub(r"//[^\n]*|/\*.*?\*/", lambda m: re.sub(r"[^\n]", " ", m.group(0)), text, flags=re.S)


def blocks(text):
    """(begin, end, header) of every brace block; the header is the statement text in front of it."""
    found, stack = [], []
    for i, c in enumerate(text):
        if c == "{":
            stack.append((i, re.split(r"[;{}]", text[max(0, i - 300):i])[-1].strip()))
        elif c == "}":
            begin, header = stack.pop()
            found.append((begin, i, header))
    assert not stack
    return found


def initialisations(text):
    """(call's place, innermost enclosing `if` block or None) of every mbar_init that a kernel makes."""
    every = blocks(text)
    for m in re.finditer(r"\bmbar_init\(", text):
        around = sorted((b for b in every if b[0] < m.start() < b[1]), key=lambda b: b[1] - b[0])
        if re.search(r"\bvoid mbar_init\($", text[max(0, m.start() - 40):m.end()]):
            continue      # the definition
        guard = next((b for b in around if b[2].startswith("if")), None)
        yield m.start(), guard


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_whoever_initialises_a_barrier_fences_it(path):
    """fence.mbarrier_init orders the executing thread's own initialisations, and the proxy fence makes them visible to the copies:
    the threads that initialise a barrier have to execute both."""
    text = without_comments(open(path).read())
    for at, guard in initialisations(text):
        line = "%s:%d" % (os.path.basename(path), text.count("\n", 0, at) + 1)
        assert guard is not None, line + ": not inside a block of the threads that initialise"
        inside = [b for b in blocks(text) if guard[0] < b[0] and b[1] < guard[1]]
        for fence in ("fence_barrier_init();", "fence_proxy_async_smem();"):
            places = [m.start() for m in re.finditer(re.escape(fence), text[:guard[1]]) if m.start() > at]
            assert any(not any(b[0] < p < b[1] for b in inside) for p in places), line + ": no " + fence


def test_the_rule_sees_every_kernel_with_barriers():
    counts = {os.path.basename(p): len(list(initialisations(without_comments(open(p).read())))) for p in SOURCES}
    for name in ("attn_bwd.cuh", "attn_paged.cuh", "attn_rope_tma.cuh", "attn_tc_pipe.cuh", "attn_tc_qtmem.cuh"):
        assert counts[name] > 0, name
