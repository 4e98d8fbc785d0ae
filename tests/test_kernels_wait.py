"""Kernels are launched while their predecessors in the stream drain: what those have written is there behind wait_previous_kernel() alone. So every kernel has that wait, and nothing in front of it
touches global memory, inputs that seldom change included: a norm's weights are what the optimiser's launch before has written. Only the sources can show it: a read that comes too early is nearly always right."""
import glob
import os
import re

import pytest

from paper_1701_06538_b200 import build as moe_build

SOURCES = sorted(glob.glob(os.path.join(moe_build.CSRC, "*.cu*")))


def closing(text, at, pair):
    """The place behind the bracket that closes the one at `at`."""
    depth = 0
    for i in range(at, len(text)):
        depth += (text[i] == pair[0]) - (text[i] == pair[1])
        if depth == 0:
            return i + 1
    raise AssertionError("no end")


def kernels(path):
    """(name, names of parameters, body) of every kernel."""
    with open(path) as f:
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    for start in re.finditer(r"__global__\s+void\s+", text):
        at = start.end()
        while True:
            m = re.compile(r"\s*(\w+)\s*\(").match(text, at)
            if m.group(1) not in ("__launch_bounds__", "__maxnreg__"):
                break
            at = closing(text, m.end() - 1, "()")
        end = closing(text, m.end() - 1, "()")
        names = re.findall(r"(\w+)\s*(?=,|$)", text[m.end():end - 1])
        brace = text.index("{", end)
        yield m.group(1), names, text[brace + 1:closing(text, brace, "{}") - 1]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_nothing_is_read_before_the_wait(path):
    for name, params, body in kernels(path):
        before, wait, _ = body.partition("wait_previous_kernel();")
        assert wait, f"{name} does not wait for the launch before it"
        before = re.sub(r'asm volatile\("prefetch\.tensormap.*', "", before)  # (maps are parameters)
        assert not re.search(r"\b(load|store|copy|fetch|atomic)\w*\s*[<(]|__ldg|(ld|st|red)\.(volatile|relaxed|global)|cp\.async|tma_|TMA", before), name
        for p in params:
            assert not re.search(rf"(?<![\w)\]] )\*\s*{p}\b|\b{p}(\.\w+|->\w+)?\s*\[|\b{p}->", before), (name, p)


def test_there_are_kernels():
    names = [n for path in SOURCES for n, _, _ in kernels(path)]
    assert len(names) > 80 and "layer_norm_kernel" in names and "newton_schulz_kernel" in names and "muon_momentum_kernel" in names
