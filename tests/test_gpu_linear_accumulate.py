"""dr_linear_wgrad with accumulate is one fp32 addition rounded to nearest, subnormals kept: in the whole blocks that the copy unit adds,
and in the columns and layouts that ordinary instructions add.  The expected value is torch's own fp32 addition, bit for bit."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen, offsets_of, strided

pytestmark = pytest.mark.gpu
F32 = torch.float32


def _check(start, n, k, sizes, dy, pad=0, shift=0):
    off, _ = offsets_of(sizes)
    x = torch.ones(sum(sizes), k, device=DEV).bfloat16()
    layer = dr.Linear(torch.zeros(len(sizes) * n, k, dtype=torch.bfloat16, device=DEV), n_groups=len(sizes))
    dw = layer.wgrad(x, dy, off)
    out, _ = strided(len(sizes) * n, k, F32, pad, shift)
    out.copy_(start)
    layer.wgrad(x, dy, off, out=out, accumulate=True)
    want = start + dw
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(out), nan)
    assert torch.equal(out[~nan].view(torch.int32), want[~nan].view(torch.int32))
    return dw, want


LAYOUTS = [(256, 256, 0, 0), (128, 208, 0, 0), (130, 200, 3, 1), (40, 16, 0, 0)]


@pytest.mark.parametrize("n,k,pad,shift", LAYOUTS)
@pytest.mark.parametrize("sizes", [[70], [3, 0, 130]], ids=str)
@pytest.mark.parametrize("scale", [0.0, 1.0, 2.0 ** -120], ids=["zero", "one", "tiny"])
def test_any_bit_pattern_plus_a_gradient(n, k, pad, shift, sizes, scale):
    g = gen(n + k)
    start = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(sizes) * n, k), device=DEV, generator=g, dtype=torch.int32).view(F32)
    start.view(-1)[::5] = torch.randint(1, 1 << 23, start.view(-1)[::5].shape, device=DEV, generator=g, dtype=torch.int32).view(F32)
    start[0, 0], start[1, 1], start[2, 2], start[3, 3] = float("nan"), float("inf"), -0.0, torch.finfo(F32).max
    dy = (torch.randn(sum(sizes), n, device=DEV, generator=g) * scale).bfloat16()
    _check(start, n, k, sizes, dy, pad, shift)


@pytest.mark.parametrize("n,k,pad,shift", LAYOUTS)
def test_sums_below_the_normal_range(n, k, pad, shift):
    start = torch.randn(n, k, device=DEV, generator=gen(3)) * 2.0 ** -128
    dw, want = _check(start, n, k, [70], torch.full((70, n), 2.0 ** -132, device=DEV).bfloat16(), pad, shift)
    assert (want.abs() < 2.0 ** -126).any()


@pytest.mark.parametrize("n,k,pad,shift", LAYOUTS)
def test_sums_at_the_top(n, k, pad, shift):
    big = torch.finfo(F32).max
    _, want = _check(torch.full((n, k), big, device=DEV), n, k, [70], torch.full((70, n), 2.0 ** 120, device=DEV).bfloat16(), pad, shift)
    assert torch.isinf(want).all()
    _, want = _check(torch.full((n, k), -big, device=DEV), n, k, [64], torch.full((64, n), 2.0 ** 121, device=DEV).bfloat16(), pad, shift)
    assert (want == 2.0 ** 127 - big).all()
