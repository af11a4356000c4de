"""What lies between the rows of strided operands (NaNs here) never enters a product: forward, both gradients, few rows and many, dense
and ragged, with contractions and widths that end inside a tile."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, check, gen, offsets_of, product, quant_weight, strided, wide_rows, wide_weight

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _padded(t, pad):
    v, _ = strided(*t.shape, t.dtype, pad, fill=float("nan"))
    v.copy_(t)
    return v


@pytest.mark.parametrize("pad", [16, 5], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("sizes,n,k", [([3], 144, 272), ([500], 272, 144), ([3, 0, 20], 144, 272), ([130, 0, 301], 272, 400), ([70, 5], 80, 48)])
def test_nans_between_rows(sizes, n, k, pad):
    groups, rows = len(sizes), sum(sizes)
    off, ends = (None, [0, rows]) if groups == 1 else offsets_of(sizes)
    g = gen(rows + n)
    x, w = torch.randn(rows, k, device=DEV, generator=g), torch.randn(groups * n, k, device=DEV, generator=g) * 0.05
    dy = torch.randn(rows, n, device=DEV, generator=g).bfloat16()
    (xq, xs), (wq, ws) = dr.quant_rows(x), quant_weight(w)
    x8, w8 = wide_rows(xq, xs), wide_weight(wq, ws)
    x, w = x.bfloat16(), w.bfloat16()
    xd, wd, dyd = x.double(), w.double(), dy.double()
    q8 = dr.Linear(_padded(wq, pad), _padded(ws, 3), n_groups=groups)
    bf = dr.Linear(_padded(w, pad), n_groups=groups)
    y8 = q8.forward(_padded(xq, pad), _padded(xs, 9), off, out_dtype=F32)
    y = bf.forward(_padded(x, pad), None, off, out_dtype=F32)
    dx = bf.dgrad(_padded(dy, pad), off, out_dtype=F32)
    dw = bf.wgrad(_padded(x, pad), _padded(dy, pad), off)
    for e in range(groups):
        lo, hi, r = ends[e], ends[e + 1], slice(e * n, (e + 1) * n)
        for name, got, a, b in (("fp8", y8[lo:hi], x8[lo:hi], w8[r].t()), ("bf16", y[lo:hi], xd[lo:hi], wd[r].t()),
                                ("dx", dx[lo:hi], dyd[lo:hi], wd[r]), ("dw", dw[r], dyd[lo:hi].t(), xd[lo:hi])):
            want, tol = product(a, b, F32)
            check(got, want, tol, f"{name} of group {e}")
