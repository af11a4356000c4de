"""Kernels that begin while the previous kernel of their stream still runs (after_previous) may read what that kernel writes: their
sources, headers included, must not load through the non-coherent path, which asks for data that nobody writes meanwhile."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22614_b200", "csrc")
INCLUDE = re.compile(r'^\s*#include\s+"([^"]+)"', re.M)
NON_COHERENT = re.compile(r"\.nc\b|__ldg\b|__ldlu\b|__restrict__")


def _text(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _reached(name, seen):
    """`name` and the project's own files that it includes."""
    if name not in seen and os.path.exists(os.path.join(CSRC, name)):
        seen.add(name)
        for inc in INCLUDE.findall(_text(name)):
            _reached(inc, seen)
    return seen


OVERLAPPED = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and re.search(r"\bafter_previous\(\)", _text(f)))


def test_there_are_such_kernels():
    assert {"quant_rows.cu", "linear_tc.cu", "linear_small.cu"} <= set(OVERLAPPED)


@pytest.mark.parametrize("source", OVERLAPPED)
def test_no_non_coherent_load(source):
    for name in sorted(_reached(source, set())):
        found = NON_COHERENT.search(_text(name))
        assert not found, f"{source} reaches {name}: {found.group(0)}"
