"""Row quantisation (dr_quant_rows) against its definition in 64 bits: codes and scales bit for bit."""
import numpy as np
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, e4m3_nearest, gen, strided

pytestmark = pytest.mark.gpu
FLT_MAX = float(np.finfo(np.float32).max)


def _want(v):
    """v fp32 [rows, cols] -> (code values, scales).  A float64 quotient of fp32 numbers rounded to fp32 equals the fp32
    quotient (53 >= 2 * 24 + 2 bits), so both roundings of the definition can be made from float64."""
    rows, cols = v.shape
    kb = -(-cols // 128)
    p = torch.nn.functional.pad(v.double(), (0, kb * 128 - cols)).view(rows, kb, 128)
    amax = torch.nan_to_num(p.abs(), nan=0.0, posinf=float("inf")).amax(2)
    s = (amax / 448).float().double().clamp(2.0 ** -126, FLT_MAX)
    q = (p / s[:, :, None]).float().double()
    return e4m3_nearest(q).view(rows, kb * 128)[:, :cols], s.t().float()


def _same(codes, scales, v):
    want, s = _want(v)
    assert torch.equal(scales, s)
    got = codes.double()
    nan = torch.isnan(v)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], want[~nan])
    assert torch.equal(torch.signbit(got[~nan]), torch.signbit(v[~nan]))  # -0 and what rounds to it keep their sign


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 127), (2, 129), (1, 4096), (33, 688), (700, 2048), (70, 257), (9, 1000)])
def test_plain(rows, cols, dtype):
    x = (torch.randn(rows, cols, device=DEV, generator=gen(rows * 7 + cols)) * torch.exp(
        torch.randn(rows, 1, device=DEV, generator=gen(1)) * 3)).to(dtype)
    if rows > 2:
        x[1] = 0
    codes, scales = dr.quant_rows(x)
    _same(codes, scales, x.float())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_special_values(dtype):
    g = gen(5)
    bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (64, 640), device=DEV, generator=g, dtype=torch.int32)
    x = bits.view(torch.float32)
    x[0, :128] = 0.0
    x[1, :128] = -0.0
    x[2, :128] = float("nan")
    x[3, 3] = float("inf")
    x[4, :128] = 1e-44   # the smallest values: the scale is held at 2^-126
    x[5, :128] = torch.finfo(torch.float32).max
    x[6, :] = 2.0 ** -133
    x = x.to(dtype)
    codes, scales = dr.quant_rows(x)
    _same(codes, scales, x.float())


@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (8, 8), (3, 0), (8, 1)])
def test_strides_and_bases(pad, shift):
    rows, cols = 37, 520
    x, _ = strided(rows, cols, torch.bfloat16, pad, shift, fill=1e30)
    x.copy_(torch.randn(rows, cols, device=DEV, generator=gen(3)).bfloat16())
    c, cbuf = strided(rows, cols, torch.uint8, pad, shift, fill=165)
    s, sbuf = strided(5, rows, torch.float32, pad, 0, fill=-7.0)
    dr.quant_rows(x, c, s)
    _same(c.contiguous().view(torch.float8_e4m3fn), s.contiguous(), x.float())
    n = rows * (cols + pad)
    c.fill_(165)
    s.fill_(-7.0)
    assert bool((cbuf == 165).all()) and bool((sbuf == -7.0).all()), f"a write outside the rows ({n})"


def test_gather_and_indices_outside():
    x = torch.randn(50, 300, device=DEV, generator=gen(4)).bfloat16()
    idx = torch.randint(50, (301,), device=DEV, generator=gen(5))
    idx[7], idx[8], idx[9] = -1, 50, 2 ** 40
    codes, scales = dr.quant_rows(x, row_index=idx)
    v = x[idx.clamp(0, 49)].float()
    v[7:10] = 0
    _same(codes, scales, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 128), (5, 688), (130, 1000), (3, 77), (2000, 768)])
def test_swiglu(rows, cols, dtype):
    x = (torch.randn(rows, 2 * cols, device=DEV, generator=gen(cols)) * 4).to(dtype)
    x[0, 0], x[0, 1], x[0, 2] = 100.0, -100.0, -88.0
    codes, scales = dr.quant_rows(x, swiglu=True)
    g, u = x.double().chunk(2, 1)
    v = g * torch.sigmoid(g) * u
    p = torch.nn.functional.pad(v, (0, -cols % 128)).view(rows, -1, 128)
    s = (p.abs().amax(2) / 448).clamp(min=2.0 ** -126).t()
    # fp32: the exponential (1 ulp), two additions or products and a division (2 ulp), the product with up: under 8 * 2^-23;
    # the scale's division adds half an ulp
    assert ((scales.double() - s).abs() <= 9 * 2.0 ** -23 * s).all()
    t = v / s.t().repeat_interleave(128, 1)[:, :cols]
    err = (codes.double() - t).abs()
    # half a step of the e4m3 grid (2^-4 relative, 2^-10 below 2^-6), and the value's own error
    assert (err <= (t.abs() * 2.0 ** -4).clamp(min=2.0 ** -10) * (1 + 1e-5) + t.abs() * 2e-6).all()
    assert codes[0, 1].item() == 0.0 or abs(v[0, 1].item() / s[0, 0].item()) > 2.0 ** -10


def test_swiglu_far_below_zero_is_not_flushed():
    x = torch.full((1, 256), -88.0, device=DEV)
    x[0, 128:] = 1e30
    codes, scales = dr.quant_rows(x, swiglu=True)
    v = -88.0 * float(torch.sigmoid(torch.tensor(-88.0, dtype=torch.float64))) * 1e30
    assert abs(scales[0, 0].item() * 448 / abs(v) - 1) < 2e-5 and (codes.float() == -448.0).all()


def test_empty_and_a_stream_of_its_own():
    codes, scales = dr.quant_rows(torch.empty(0, 256, dtype=torch.bfloat16, device=DEV))
    assert codes.shape == (0, 256) and scales.shape == (2, 0)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        x = torch.randn(4096, 2048, device=DEV, generator=gen(9))
        codes, scales = dr.quant_rows(x)
    st.synchronize()
    _same(codes, scales, x)


def test_graph_replay_reads_the_new_values():
    x = torch.randn(64, 512, device=DEV, generator=gen(1))
    codes, scales = dr.quant_rows(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dr.quant_rows(x, codes, scales)
    x.mul_(3.5)
    graph.replay()
    torch.cuda.synchronize()
    _same(codes, scales, x)
