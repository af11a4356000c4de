"""Child process of the tests of the linear layers' bounded waits: the counter that it raises is the process's own.

    python linear_waits_worker.py give_up | counted_at_once | long_contractions
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen, offsets_of, quant_weight

BF16, F32 = torch.bfloat16, torch.float32


def count():
    rc, n = dr.dr_diag_linear_wait_failures()
    assert rc == 0
    return n


def calls():
    """Every tensor-core kernel in its forms: few rows with and without a split contraction, pairs of CTAs, dense and ragged, gradients."""
    for sizes, n, k in (([5], 256, 1024), ([40], 8192, 512), ([300], 512, 512), ([3, 0, 60, 17], 384, 512), ([600, 0, 301], 384, 512)):
        groups, rows = len(sizes), sum(sizes)
        off = None if groups == 1 else offsets_of(sizes)[0]
        x = torch.randn(rows, k, device=DEV, generator=gen(rows)).bfloat16()
        dy = torch.randn(rows, n, device=DEV, generator=gen(n)).bfloat16()
        w = torch.randn(groups * n, k, device=DEV, generator=gen(k)) * 0.05
        bf, q8 = dr.Linear(w.bfloat16(), n_groups=groups), dr.Linear(*quant_weight(w), n_groups=groups)
        xq, xs = dr.quant_rows(x)
        name = f"{sizes} x {n} x {k}"
        yield f"bf16 {name}", lambda out: bf.forward(x, None, off, out=out), (rows, n, BF16)
        yield f"fp8 {name}", lambda out: q8.forward(xq, xs, off, out=out), (rows, n, BF16)
        yield f"dgrad {name}", lambda out: bf.dgrad(dy, off, out=out), (rows, k, BF16)
        yield f"wgrad {name}", lambda out: bf.wgrad(x, dy, off, out=out), (groups * n, k, F32)


def give_up():
    """Without its copies a kernel gives up, says so, and leaves a device on which the next call is right."""
    assert dr.dr_diag_linear_waits(2000001, 0) < 0 and dr.dr_diag_linear_waits(0, 2) < 0
    for name, call, (rows, cols, dtype) in calls():
        want = call(torch.empty(rows, cols, dtype=dtype, device=DEV)).clone()
        torch.cuda.synchronize()
        before = count()
        got = torch.full((rows, cols), 9.0, dtype=dtype, device=DEV)
        assert dr.dr_diag_linear_waits(20000, 1) == 0
        call(got)
        assert dr.dr_diag_linear_waits(0, 0) == 0
        torch.cuda.synchronize()
        after = count()
        assert after > before, f"{name}: no wait ran out"
        assert (got[:3] == 9.0).all(), f"{name}: an output without operands"
        call(got)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and count() == after, f"{name}: the next call"
        print(name, after - before, flush=True)
    assert before > 0


def counted_at_once():
    """The counter read right behind a call on a stream of its own, which the default stream does not wait for."""
    side = torch.cuda.Stream()
    for name, call, (rows, cols, dtype) in calls():
        out = torch.zeros(rows, cols, dtype=dtype, device=DEV)
        torch.cuda.synchronize()
        before = count()
        assert dr.dr_diag_linear_waits(50000, 1) == 0
        with torch.cuda.stream(side):
            call(out)
        assert dr.dr_diag_linear_waits(0, 0) == 0
        assert count() > before, f"{name}: read too early"


def long_contractions():
    """A tile that takes many times the limit's fixed part (1 ms here, 2 s in earnest, where the contraction may be 2^25 steps long):
    the limit has to grow with the contraction.  All other values are zero, so the result shows whether the last step was taken."""
    def of(rows, cols, step):
        """Zeros, and ones in the first and last positions of the contraction (along the rows or along the columns)."""
        t = torch.zeros(rows, cols, dtype=BF16, device=DEV)
        for at in (0, -1):
            (t[at] if step == "rows" else t[:, at]).fill_(1)
        return t

    long = 1 << 23
    layer = dr.Linear(torch.zeros(64, 64, dtype=BF16, device=DEV))
    x, dy = of(long, 64, "rows"), of(long, 64, "rows")
    wide = dr.Linear(of(128, long, "cols"))
    few, many = of(4, long, "cols"), of(100, long, "cols")
    back = dr.Linear(of(long, 64, "rows"))
    gy = of(100, long, "cols")
    for name, call in (("wgrad", lambda: layer.wgrad(x, dy)), ("few rows", lambda: wide.forward(few, out_dtype=F32)),
                       ("many rows", lambda: wide.forward(many, out_dtype=F32)), ("dgrad", lambda: back.dgrad(gy, out_dtype=F32))):
        assert dr.dr_diag_linear_waits(1000, 0) == 0
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        got = call()
        b.record()
        assert dr.dr_diag_linear_waits(0, 0) == 0
        assert count() == 0, f"{name}: a wait ran out"
        assert (got == 2).all(), name
        print(f"{name}: {a.elapsed_time(b):.1f} ms", flush=True)
        assert a.elapsed_time(b) > 2.0, "too short a contraction to show anything"


if __name__ == "__main__":
    {"give_up": give_up, "counted_at_once": counted_at_once, "long_contractions": long_contractions}[sys.argv[1]]()
    print("done")
