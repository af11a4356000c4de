"""Child process of the test of the attention kernels' bounded waits: the counter that it raises is the process's own."""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

import paper_2607_22614_b200 as dr
from attend_util import make_cache, make_table
from linear_util import DEV, gen


def count():
    rc, n = dr.dr_diag_linear_wait_failures()
    assert rc == 0
    return n


def main():
    """Without its copies a kernel gives up, says so, and leaves a device on which the next call is right."""
    for dim in (64, 128):
        for lengths, added in (([300, 40], [1, 1]), ([2000, 700], [1, 1]), ([900, 70], [3, 2]), ([900, 170], [300, 150]), ([900, 170], [70, 1])):
            g = gen(dim)
            cache = dr.KVCache(*make_cache(g, 60, 2, 64, dim))
            table = make_table(g, lengths, 64, 60, 40 if max(lengths) > 500 else 5)
            offsets = torch.tensor([0, added[0], sum(added)], dtype=torch.int32, device=DEV)
            q = torch.randn(sum(added), 8 * dim, device=DEV, generator=g).bfloat16()
            L = torch.tensor(lengths, dtype=torch.int32, device=DEV)
            want = cache.attend(q, L, table, offsets)
            torch.cuda.synchronize()
            before, out = count(), torch.full_like(want, 9.0)
            assert dr.dr_diag_linear_waits(20000, 1) == 0
            cache.attend(q, L, table, offsets, out=out)
            assert dr.dr_diag_linear_waits(0, 0) == 0
            torch.cuda.synchronize()
            after = count()
            assert after > before, f"{dim} {lengths} {added}: no wait ran out"
            cache.attend(q, L, table, offsets, out=out)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and count() == after, f"{dim} {lengths} {added}: the next call"
            print(dim, lengths, added, after - before, flush=True)


if __name__ == "__main__":
    main()
    print("done")
