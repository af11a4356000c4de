"""Many groups and skewed ones: the running sums across many warps' worth of groups, the step from 512 groups (tensor cores) to 513 (plain
kernel), and batches whose average is a few rows a group while one group holds most of them."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, check, gen, offsets_of, product, quant_weight, wide_rows, wide_weight

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _sizes(groups, kind):
    """Rows of each group: `few`, a handful here and there; `many`, more than 64 on average, empty groups among them; `one`, nearly all rows in one
    group, fewer than 64 on average."""
    g = torch.Generator().manual_seed(groups)
    if kind == "few":
        return torch.randint(0, 5, (groups,), generator=g).tolist()
    if kind == "many":
        return (torch.randint(0, 200, (groups,), generator=g) * (torch.rand(groups, generator=g) < 0.8)).tolist()
    s = torch.randint(0, 2, (groups,), generator=g)
    s[groups * 2 // 3] = 40 * groups - 7
    return s.tolist()


@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
@pytest.mark.parametrize("kind", ["few", "many", "one"])
@pytest.mark.parametrize("groups", [31, 32, 33, 100, 128, 511, 512, 513])
def test_forward(groups, kind, fp8):
    n, k = (40, 144) if groups > 128 else (200, 272)
    sizes = _sizes(groups, kind)
    off, ends = offsets_of(sizes, lead=1)
    rows, g = sum(sizes) + 4, gen(groups)
    x = torch.randn(rows, k, device=DEV, generator=g)
    w = torch.randn(groups * n, k, device=DEV, generator=g) * 0.05
    if fp8:
        (xq, xs), (wq, ws) = dr.quant_rows(x), quant_weight(w)
        xd, wd = wide_rows(xq, xs), wide_weight(wq, ws)
    else:
        xq, xs, wq, ws = x.bfloat16(), None, w.bfloat16(), None
        xd, wd = xq.double(), wq.double()
    y = torch.full((rows, n), -77.0, device=DEV)
    dr.Linear(wq, ws, n_groups=groups).forward(xq, xs, off, out=y)
    assert (y[:1] == -77.0).all() and (y[ends[-1]:] == -77.0).all()
    for e in range(groups):
        lo, hi = ends[e], ends[e + 1]
        if lo < hi:
            want, tol = product(xd[lo:hi], wd[e * n:(e + 1) * n].t(), F32)
            check(y[lo:hi], want, tol, f"group {e}")


@pytest.mark.parametrize("kind", ["few", "many", "one"])
@pytest.mark.parametrize("groups", [33, 128, 512, 513])
def test_gradients(groups, kind):
    n, k = (40, 144) if groups > 128 else (200, 272)
    sizes = _sizes(groups, kind)
    off, ends = offsets_of(sizes, lead=1)
    rows, g = sum(sizes) + 4, gen(groups)
    x = torch.randn(rows, k, device=DEV, generator=g).bfloat16()
    dy = torch.randn(rows, n, device=DEV, generator=g).bfloat16()
    w = (torch.randn(groups * n, k, device=DEV, generator=g) * 0.05).bfloat16()
    for t in (x, dy):
        t[:1] = float("nan")
        t[ends[-1]:] = float("inf")
    xd, dyd, wd = x.double(), dy.double(), w.double()
    layer = dr.Linear(w, n_groups=groups)
    dx = torch.full((rows, k), -77.0, device=DEV)
    layer.dgrad(dy, off, out=dx)
    dw = torch.full((groups * n, k), float("nan"), device=DEV)
    layer.wgrad(x, dy, off, out=dw)
    assert (dx[:1] == -77.0).all() and (dx[ends[-1]:] == -77.0).all()
    for e in range(groups):
        lo, hi, r = ends[e], ends[e + 1], slice(e * n, (e + 1) * n)
        want, tol = product(dyd[lo:hi], wd[r], F32)
        check(dx[lo:hi], want, tol, f"dx of group {e}")
        want, tol = product(dyd[lo:hi].t(), xd[lo:hi], F32)
        check(dw[r], want, tol, f"dw of group {e}")
