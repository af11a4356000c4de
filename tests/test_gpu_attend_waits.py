"""The bounded waits of the attention kernels, in a child process of their own (the counter of waits that ran out stays 0 in this one)."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_kernels_that_give_up_say_so_and_leave_the_device_usable():
    worker = os.path.join(os.path.dirname(os.path.abspath(__file__)), "attend_waits_worker.py")
    p = subprocess.run([sys.executable, worker], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.rstrip().endswith("done"), p.stdout[-2000:] + p.stderr[-2000:]
