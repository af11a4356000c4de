"""fp8 products whose scales lie at the ends of fp32, by the formula: the sum of a block of 128 times the product of its two scales,
rounded once.  Aligned operands and operands that no tensor map can read have to agree with it alike."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, check, gen, quant_weight, strided

pytestmark = pytest.mark.gpu
F32 = torch.float32


def _by_formula(xq, xs, wq, ws):
    """The product in 64 bits from the fp32 products of scales, and the error that fp32 sums of it may have in any order: every term
    is multiplied and added at most (k + 3) times with 2^-23 each."""
    k, n = xq.shape[1], wq.shape[0]
    y = torch.zeros(xq.shape[0], n, dtype=torch.float64, device=DEV)
    mass = y.clone()
    for b in range(-(-k // 128)):
        f = (xs[b][:, None] * ws[torch.arange(n, device=DEV) // 128, b][None, :]).double()
        x, w = xq[:, 128 * b:128 * b + 128].double(), wq[:, 128 * b:128 * b + 128].double()
        y += f * (x @ w.t())
        mass += f * (x.abs() @ w.abs().t())
    return y, (k + 3) * 2.0 ** -23 * mass + 1e-37


def _codes(rows, cols, g, most):
    return (torch.rand(rows, cols, device=DEV, generator=g) * 2 * most - most).to(torch.float8_e4m3fn)


# the product of the scales is ordinary, a code times its own scale is not a finite or not a normal number
@pytest.mark.parametrize("x_scale,w_scale", [(3e38, 1e-36), (1e-36, 3e38), (2.0 ** 127, 2.0 ** -126), (2.0 ** -120, 2.0 ** 100)])
@pytest.mark.parametrize("pad", [16, 3], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("rows,n,k", [(5, 200, 400), (300, 130, 272)])
def test_extreme_scales(rows, n, k, pad, x_scale, w_scale):
    g = gen(rows + k)
    xq, _ = strided(rows, k, torch.float8_e4m3fn, pad)
    wq, _ = strided(n, k, torch.float8_e4m3fn, pad)
    xq.copy_(_codes(rows, k, g, 6))
    wq.copy_(_codes(n, k, g, 6))
    blocks = -(-k // 128)
    xs = x_scale * (0.5 + 0.5 * torch.rand(blocks, rows, device=DEV, generator=g))
    ws = w_scale * (0.5 + 0.5 * torch.rand(-(-n // 128), blocks, device=DEV, generator=g))
    y = dr.Linear(wq, ws).forward(xq, xs, out_dtype=F32)
    want, tol = _by_formula(xq, xs, wq, ws)
    assert torch.isfinite(want).all() and want.abs().max() < 3e38
    check(y, want, tol)


@pytest.mark.parametrize("pad", [16, 3], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("rows", [5, 300])
def test_a_row_that_holds_an_infinity(rows, pad):
    """Its scale is FLT_MAX and its code 448; with a small weight there the result is a finite number."""
    n, k, g = 130, 400, gen(rows)
    x = torch.randn(rows, k, device=DEV, generator=g)
    x[1, 7] = float("inf")
    w = torch.randn(n, k, device=DEV, generator=g) * 1e-30
    w[:, 7] = 0
    w[3, 7] = 4e-33
    q, ws = quant_weight(w)
    s, scales = dr.quant_rows(x)
    xq, _ = strided(rows, k, torch.float8_e4m3fn, pad)
    wq, _ = strided(n, k, torch.float8_e4m3fn, pad)
    xq.copy_(s)
    wq.copy_(q)
    assert scales[0, 1] == torch.finfo(F32).max and xq[1, 7].float() == 448
    y = dr.Linear(wq, ws).forward(xq, scales, out_dtype=F32)
    want, tol = _by_formula(xq, scales, wq, ws)
    assert want[1, 3].abs() > 1 and torch.isfinite(y).all()
    check(y, want, tol)
