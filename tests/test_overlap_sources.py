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


# Ordinary shared memory that passes between CTAs of a cluster: the sums that few rows' CTAs exchange (written by the others, read
# here, written again), and the rows that wgrad clears before the other CTA issues the products.
CLUSTER_SCOPE = [("linear_small.cu", r"bar_wait<true>\([^;]*sums_empty", 1), ("linear_small.cu", r"bar_wait<true>\([^;]*sums_full", 1),
                 ("linear_small.cu", r"bar_arrive_cluster\([^;]*sums_empty[^;]*, true\)", 1),
                 ("linear_tc.cu", r"bar_arrive_cluster\(full[^;]*, valid < 64\)", 1), ("linear_tc.cu", r"warp_wait<OP == kWgrad>\(full", 1),
                 ("tc_ptx.cuh", r"mbarrier\.arrive\.release\.cluster", 1), ("tc_ptx.cuh", r"mbarrier\.try_wait\.parity\.acquire\.cluster", 1)]


@pytest.mark.parametrize("name,form,times", CLUSTER_SCOPE)
def test_memory_handed_to_another_cta_is_released_and_acquired_at_cluster_scope(name, form, times):
    assert len(re.findall(form, _text(name))) == times
