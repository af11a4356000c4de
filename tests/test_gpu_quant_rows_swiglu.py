"""The error of the SwiGLU form against 64 bits, beside that of the elementary fp32 form g / (1 + exp(-g)) * u with every step rounded
to nearest.  Rows of one column: the scale is the value's magnitude over 448, and its sign is the code's."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spread", [1.0, 4.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_less_exact_than_the_elementary_form(dtype, spread):
    n = 1 << 20
    x = (torch.randn(n, 2, device=DEV, generator=gen(7)) * spread).to(dtype)
    codes, scales = dr.quant_rows(x, swiglu=True)
    g, u = x.double().unbind(1)
    want = g * torch.sigmoid(g) * u / 448
    f, v = x.float().unbind(1)
    plain = ((f / (1 + torch.exp(-f)) * v).double() / 448).float()
    keep = want.abs() > 2.0 ** -120
    got = scales[0] * codes[:, 0].float().sign()

    def error(a):
        return ((a.double() - want) / want)[keep] * 2.0 ** 24

    mine, other = error(got), error(plain)
    assert mine.square().mean().sqrt() <= other.square().mean().sqrt()
    assert mine.abs().max() <= 9 * 2.0  # the bound of the row quantisation tests, 9 * 2^-23


def test_ends_of_the_range():
    """Gates far out, infinities and NaNs: silu(g) * u as IEEE arithmetic of the definition gives it."""
    inf, nan, big = float("inf"), float("nan"), torch.finfo(torch.float32).max
    rows = [(inf, 2.0, inf), (-inf, 2.0, nan), (nan, 1.0, nan), (1.0, nan, nan), (big, 0.5, big / 2), (-big, 1.0, 0.0), (-1e30, 1e30, 0.0),
            (1e30, 1e30, inf), (-200.0, big, 0.0), (0.0, 5.0, 0.0), (-0.0, 5.0, 0.0), (inf, 0.0, nan), (100.0, 3.0, 300.0)]
    x = torch.tensor([[g, u] for g, u, _ in rows], device=DEV)
    codes, scales = dr.quant_rows(x, swiglu=True)
    for i, (g, u, v) in enumerate(rows):
        c, s = codes[i, 0].float().item(), scales[0, i].item()
        if v != v:
            assert c != c and s == 2.0 ** -126, (g, u)   # a NaN is skipped by the maximum and keeps its code
        elif v == 0:
            assert c == 0 and s == 2.0 ** -126, (g, u)
        elif v == inf:
            assert c == 448 and s == big, (g, u)
        else:
            assert c == 448 and abs(s * 448 / v - 1) < 2e-6, (g, u)
