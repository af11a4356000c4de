"""The bounded waits of the linear layers' tensor-core kernels, in a child process of their own (the counter of waits that ran out
stays 0 in this one)."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
WORKER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "linear_waits_worker.py")


def _run(part):
    p = subprocess.run([sys.executable, WORKER, part], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.rstrip().endswith("done"), p.stdout[-2000:] + p.stderr[-2000:]


def test_kernels_that_give_up_say_so_and_leave_the_device_usable():
    _run("give_up")


def test_the_counter_waits_for_every_stream():
    _run("counted_at_once")


def test_the_limit_grows_with_the_contraction():
    _run("long_contractions")
