"""Linear layers over rollout weights (dr_linear_*) against plain 64-bit products: types, ragged groups, strides, odd
sizes, masked rows that hold infinities, gradients against the formula and against differences."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, check, gen, offsets_of, product, quant_weight, strided, wide_rows, wide_weight

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _inputs(rows, n, k, groups, fp8, seed=0):
    g = gen(seed + 1000 * rows + n)
    x = torch.randn(rows, k, device=DEV, generator=g)
    if rows > 3:
        x[2] = 0
    w = torch.randn(groups * n, k, device=DEV, generator=g) * 0.05
    if fp8:
        xq, xs = dr.quant_rows(x)
        wq, ws = quant_weight(w)
        return xq, xs, wq, ws, wide_rows(xq, xs), wide_weight(wq, ws)
    x, w = x.bfloat16(), w.bfloat16()
    return x, None, w, None, x.double(), w.double()


DENSE = [(1, 128, 128), (1, 1376, 256), (2, 130, 208), (5, 256, 688), (7, 130, 200), (16, 512, 2064), (17, 144, 1024), (33, 640, 512),
         (64, 384, 4096), (65, 257, 384), (128, 256, 128), (129, 272, 720), (300, 528, 1040), (257, 1024, 64), (520, 1376, 256),
         (1025, 768, 144), (40, 16, 16), (3, 1, 1), (9, 12, 10), (200, 136, 24), (1, 4096, 12288)]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
@pytest.mark.parametrize("rows,n,k", DENSE)
def test_dense(rows, n, k, fp8, out):
    xq, xs, wq, ws, xd, wd = _inputs(rows, n, k, 1, fp8)
    y = dr.Linear(wq, ws).forward(xq, xs, out_dtype=out)
    want, tol = product(xd, wd.t(), out)
    check(y, want, tol)


GROUPED = [([3, 0, 1, 7], 256, 256), ([0, 0, 130, 0, 1, 64, 0, 259], 384, 512), ([1] * 33, 144, 272), ([0, 300, 0], 192, 208),
           ([5, 17, 33, 2, 90], 128, 1040), ([128, 128, 256], 512, 128), ([2, 0, 9], 40, 64), ([31, 1, 140], 12, 24),
           ([0, 0, 0], 128, 128), ([70, 200, 500, 40], 1536, 768), ([600, 0, 1300, 513], 384, 528), ([1100, 901], 144, 256),
           ([513, 2000, 30], 40, 128)]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
@pytest.mark.parametrize("sizes,n,k", GROUPED)
def test_grouped(sizes, n, k, fp8, out):
    lead, rows, groups = 3, 3 + sum(sizes) + 5, len(sizes)
    off, ends = offsets_of(sizes, lead)
    xq, xs, wq, ws, xd, wd = _inputs(rows, n, k, groups, fp8)
    if fp8:  # rows that no group owns hold NaN codes and infinite scales
        xq.view(torch.uint8)[:lead] = 0x7F
        xs[:, -5:] = float("inf")
    else:
        xq[:lead] = float("nan")
        xq[-5:] = float("inf")
    y = torch.full((rows, n), -77.0, dtype=out, device=DEV)
    dr.Linear(wq, ws, n_groups=groups).forward(xq, xs, off, out=y)
    assert (y[:lead] == -77.0).all() and (y[ends[-1]:] == -77.0).all(), "a row that no group owns was written"
    for e in range(groups):
        lo, hi = ends[e], ends[e + 1]
        want, tol = product(xd[lo:hi], wd[e * n:(e + 1) * n].t(), out)
        check(y[lo:hi], want, tol, f"group {e}")


@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
def test_infinities_stay_in_their_rows_and_columns(fp8):
    sizes, n, k = [40, 3, 90], 256, 384
    off, ends = offsets_of(sizes)
    xq, xs, wq, ws, xd, wd = _inputs(sum(sizes), n, k, 3, fp8)
    if fp8:
        xq.view(torch.uint8)[41, 5] = 0x7F
        wq.view(torch.uint8)[n + 7, 9] = 0x7F   # expert 1, feature 7
    else:
        xq[41, 5] = float("nan")
        wq[n + 7, 9] = float("inf")
    y = dr.Linear(wq, ws, n_groups=3).forward(xq, xs, off, out_dtype=F32)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[41] = True
    want[40:43, 7] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
@pytest.mark.parametrize("pad,shift", [(16, 0), (16, 16), (8, 0), (3, 0), (16, 1)])
def test_strides_and_bases(pad, shift, fp8):
    sizes, n, k = [30, 0, 101], 272, 400
    off, ends = offsets_of(sizes)
    rows = sum(sizes)
    xq, xs, wq, ws, xd, wd = _inputs(rows, n, k, 3, fp8)
    xv, _ = strided(rows, k, xq.dtype, pad, shift)
    xv.copy_(xq)
    wv, _ = strided(3 * n, k, wq.dtype, pad, shift)
    wv.copy_(wq)
    sv = None
    if fp8:
        sv, _ = strided(ws.shape[0], ws.shape[1], F32, 5, 3)
        sv.copy_(ws)
        xsv, _ = strided(xs.shape[0], rows, F32, 7, 1)
        xsv.copy_(xs)
        xs = xsv
    for out in (BF16, F32):
        yv, ybuf = strided(rows, n, out, pad, shift, fill=9.0)
        dr.Linear(wv, sv, n_groups=3).forward(xv, xs, off, out=yv)
        for e in range(3):
            lo, hi = ends[e], ends[e + 1]
            want, tol = product(xd[lo:hi], wd[e * n:(e + 1) * n].t(), out)
            check(yv[lo:hi], want, tol, f"group {e}")
        yv.fill_(9.0)
        assert (ybuf == 9.0).all(), "a write outside the rows"


def test_offsets_out_of_range_stay_inside():
    n, k = 128, 256
    xq, xs, wq, ws, xd, wd = _inputs(50, n, k, 4, True)
    off = torch.tensor([-5, 10, 4, 30, 1000], dtype=torch.int32, device=DEV)  # group 0: 0..10, 1: none, 2: 4..30, 3: 30..50
    ybuf = torch.full((60, n), 9.0, device=DEV)
    dr.Linear(wq, ws, n_groups=4).forward(xq, xs, off, out=ybuf[5:55])
    assert (ybuf[:5] == 9.0).all() and (ybuf[55:] == 9.0).all()
    want, tol = product(xd[30:], wd[3 * n:].t(), F32)
    check(ybuf[35:55], want, tol)
    want, tol = product(xd[:4], wd[:n].t(), F32)
    check(ybuf[5:9], want, tol)


GRADS = [([40], 256, 256), ([3, 0, 1, 7], 256, 384), ([0, 0, 130, 0, 1, 64, 0, 259], 384, 512), ([1] * 33, 144, 272),
         ([0, 300, 0], 192, 208), ([63, 64, 65, 66], 128, 136), ([2, 0, 9], 40, 64), ([31, 1, 140], 12, 24), ([0, 0, 0], 128, 128),
         ([7, 20], 130, 201), ([600, 70], 1536, 768), ([1, 2, 1, 90, 0, 7, 90, 2, 1, 0, 64] * 3, 544, 192), ([3, 0, 65] * 9, 400, 656),
         ([1, 0, 2] * 11, 896, 304)]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("sizes,n,k", GRADS)
def test_gradients(sizes, n, k, out):
    lead, rows, groups = 2, 2 + sum(sizes) + 3, len(sizes)
    off, ends = offsets_of(sizes, lead)
    x, _, w, _, xd, wd = _inputs(rows, n, k, groups, False)
    dy = (torch.randn(rows, n, device=DEV, generator=gen(n)) * 0.1).bfloat16()
    for t in (x, dy):
        t[:lead] = float("nan")
        t[ends[-1]:] = float("inf")
    xd, dyd = x.double(), dy.double()
    layer = dr.Linear(w, n_groups=groups)
    dx = torch.full((rows, k), -77.0, dtype=out, device=DEV)
    layer.dgrad(dy, off, out=dx)
    dw = torch.full((groups * n, k), float("nan"), device=DEV)
    layer.wgrad(x, dy, off, out=dw)
    assert (dx[:lead] == -77.0).all() and (dx[ends[-1]:] == -77.0).all()
    start = torch.randn(groups * n, k, device=DEV, generator=gen(3))
    acc = start.clone()
    layer.wgrad(x, dy, off, out=acc, accumulate=True)
    for e in range(groups):
        lo, hi, r = ends[e], ends[e + 1], slice(e * n, (e + 1) * n)
        want, tol = product(dyd[lo:hi], wd[r], out)
        check(dx[lo:hi], want, tol, f"dx of group {e}")
        want, tol = product(dyd[lo:hi].t(), xd[lo:hi], F32)
        check(dw[r], want, tol, f"dw of group {e}")
        check(acc[r], want + start[r].double(), tol + 2.0 ** -23 * (want.abs() + start[r].abs()), f"accumulated dw of group {e}")


@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (4, 0), (3, 0), (8, 1)])
def test_gradient_strides_and_bases(pad, shift):
    sizes, n, k = [30, 0, 101], 272, 400
    off, ends = offsets_of(sizes)
    rows = sum(sizes)
    x, _, w, _, xd, wd = _inputs(rows, n, k, 3, False)
    dy = torch.randn(rows, n, device=DEV, generator=gen(8)).bfloat16()

    def moved(t):
        v, _ = strided(*t.shape, t.dtype, pad, shift)
        v.copy_(t)
        return v

    layer = dr.Linear(moved(w), n_groups=3)
    dx, dxbuf = strided(rows, k, BF16, pad, shift, fill=9.0)
    dw, dwbuf = strided(3 * n, k, F32, pad, shift, fill=9.0)
    layer.dgrad(moved(dy), off, out=dx)
    layer.wgrad(moved(x), moved(dy), off, out=dw)
    for e in range(3):
        lo, hi, r = ends[e], ends[e + 1], slice(e * n, (e + 1) * n)
        want, tol = product(dy.double()[lo:hi], wd[r], BF16)
        check(dx[lo:hi], want, tol)
        want, tol = product(dy.double()[lo:hi].t(), xd[lo:hi], F32)
        check(dw[r], want, tol)
    dx.fill_(9.0)
    dw.fill_(9.0)
    assert (dxbuf == 9.0).all() and (dwbuf == 9.0).all(), "a write outside the rows"


def test_gradients_against_differences():
    """The loss sum(y * dy) is linear in x and in w, so a central difference has no truncation error.  All values are multiples
    of 1/8 (of 1/64 for products) below 2^8 in magnitude: fp32 sums of them are exact, and so is the comparison."""
    sizes, n, k = [9, 0, 21], 48, 64
    off, _ = offsets_of(sizes)
    rows, g = sum(sizes), gen(11)

    def eighths(*shape):
        return (torch.randint(-8, 9, shape, device=DEV, generator=g) / 8).bfloat16()

    x, w, dy = eighths(rows, k), eighths(3 * n, k), eighths(rows, n)
    layer = dr.Linear(w, n_groups=3)
    dx = layer.dgrad(dy, off, out_dtype=F32)
    dw = layer.wgrad(x, dy, off)

    def loss(xx, ww):
        y = dr.Linear(ww, n_groups=3).forward(xx, None, off, out_dtype=F32)
        return (y.double() * dy.double()).sum().item()

    h = 0.125
    for r, c in [(0, 0), (8, 63), (9, 5), (29, 40), (15, 17)]:
        up, down = x.clone(), x.clone()
        up[r, c] += h
        down[r, c] -= h
        assert (loss(up, w) - loss(down, w)) / (2 * h) == dx[r, c].item()
    for r, c in [(0, 0), (47, 63), (60, 3), (100, 40), (143, 63)]:
        up, down = w.clone(), w.clone()
        up[r, c] += h
        down[r, c] -= h
        assert (loss(x, up) - loss(x, down)) / (2 * h) == dw[r, c].item()


@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
def test_same_call_same_bits_on_any_stream_and_in_a_graph(fp8):
    sizes, n, k = [200, 0, 17, 3], 512, 1024
    off, _ = offsets_of(sizes)
    xq, xs, wq, ws, _, _ = _inputs(sum(sizes), n, k, 4, fp8)
    layer = dr.Linear(wq, ws, n_groups=4)
    dy = torch.randn(sum(sizes), n, device=DEV, generator=gen(2)).bfloat16()

    def run():
        got = [layer.forward(xq, xs, off)]
        if not fp8:
            got += [layer.dgrad(dy, off), layer.wgrad(xq, dy, off)]
        return got

    first = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = []
    for st in streams:
        with torch.cuda.stream(st):
            both.append([run() for _ in range(3)])
    torch.cuda.synchronize()
    for got in (g for b in both for g in b):
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    out = [torch.zeros_like(t) for t in first]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(xq, xs, off, out=out[0])
        if not fp8:
            layer.dgrad(dy, off, out=out[1])
            layer.wgrad(xq, dy, off, out=out[2])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    # the graph reads offsets on the device: other sizes, same launch
    off.copy_(torch.tensor([0, 10, 150, 215, 220], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    again = run()
    assert all(torch.equal(a, b) for a, b in zip(again, out))


def test_no_rows():
    w = torch.randn(256, 128, device=DEV).bfloat16()
    layer = dr.Linear(w, n_groups=2)
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    x, dy = torch.empty(0, 128, dtype=BF16, device=DEV), torch.empty(0, 128, dtype=BF16, device=DEV)
    assert layer.forward(x, None, off).shape == (0, 128) and layer.dgrad(dy, off).shape == (0, 128)
    dw = torch.full((256, 128), 3.0, device=DEV)
    layer.wgrad(x, dy, off, out=dw, accumulate=True)
    assert (dw == 3.0).all()
    layer.wgrad(x, dy, off, out=dw)
    assert (dw == 0.0).all()


def test_arena_weights():
    """A layer taken from an arena that dr_reshard has written, dense and by expert, bf16 and fp8."""
    from synth.configs import MID
    for spec, leaf in ((MID[0]["spec"], "down"), (MID[2]["spec"], "w13")):
        for dtype in (dr.DR_BF16, dr.DR_FP8_E4M3_B128):
            plan = dr.Plan(spec, dtype=dtype)
            flat = torch.randn(plan.info.src_bytes // 4, device=DEV, generator=gen(1)) * 0.02
            arena = torch.empty(plan.info.dst_bytes, dtype=torch.uint8, device=DEV)
            plan.reshard(flat, arena)
            layer = plan.linear(arena, "layers.1." + leaf)
            assert layer.n_groups == max(1, spec["n_experts"] if leaf == "w13" else 1)
            x = torch.randn(10, layer.in_features, device=DEV, generator=gen(2))
            off = None if layer.n_groups == 1 else offsets_of([2, 0, 5, 0, 0, 1, 0, 2])[0]
            xq, xs = dr.quant_rows(x) if layer.fp8 else (x.bfloat16(), None)
            y = layer.forward(xq, xs, off, out_dtype=F32)
            wd = wide_weight(layer.weight, layer.scale) if layer.fp8 else layer.weight.double()
            xd = wide_rows(xq, xs) if layer.fp8 else xq.double()
            ends = [0, 10] if off is None else off.tolist()
            for e in range(layer.n_groups):
                lo, hi = ends[e], ends[e + 1]
                want, tol = product(xd[lo:hi], wd[e * layer.out_features:(e + 1) * layer.out_features].t(), F32)
                check(y[lo:hi], want, tol)


def test_refusals_with_a_device():
    B = dr.binding
    w = torch.zeros(256, 128, dtype=BF16, device=DEV)
    layer = dr.Linear(w, n_groups=2)
    x, y = torch.zeros(4, 128, dtype=BF16, device=DEV), torch.zeros(4, 128, dtype=BF16, device=DEV)
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    p, q, o, h = x.data_ptr(), y.data_ptr(), off.data_ptr(), layer.handle
    f = B.dr_linear_forward
    assert f(None, p, 128, None, 0, 4, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert f(h, p, 128, None, 0, 4, None, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID      # offsets missing
    assert f(h, p, 127, None, 0, 4, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert f(h, p, 128, None, 0, 4, o, q, 127, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert f(h, p, 128, p, 4, 4, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID            # scales for a bf16 layer
    assert f(h, None, 128, None, 0, 4, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert f(h, p, 128, None, 0, 4, o, q, 128, dr.DR_FP8_E4M3_B128, None) == B.DR_ERR_UNSUPPORTED
    assert f(h, p, 128, None, 0, 1 << 31, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_UNSUPPORTED
    assert f(h, p + 1, 128, None, 0, 4, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_ALIGN
    assert f(h, p, 128, None, 0, 4, o + 2, q, 128, dr.DR_BF16, None) == B.DR_ERR_ALIGN
    assert f(h, p, 128, None, 0, 4, o, q + 2, 128, dr.DR_F32, None) == B.DR_ERR_ALIGN
    assert B.dr_linear_dgrad(h, p, 100, 4, o, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert B.dr_linear_wgrad(h, p, 128, q, 128, 4, o, None, 128, 0, None) == B.DR_ERR_INVALID
    assert B.dr_linear_wgrad(h, p, 128, q, 128, 4, o, w.data_ptr(), 128, 2, None) == B.DR_ERR_INVALID
    q8 = dr.Linear(torch.zeros(128, 128, dtype=torch.float8_e4m3fn, device=DEV), torch.ones(1, 1, device=DEV))
    assert f(q8.handle, p, 128, None, 0, 4, None, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID     # scales missing
    assert f(q8.handle, p, 128, p, 3, 4, None, q, 128, dr.DR_BF16, None) == B.DR_ERR_INVALID        # ld_scale < rows
    assert B.dr_linear_dgrad(q8.handle, p, 128, 4, None, q, 128, dr.DR_BF16, None) == B.DR_ERR_UNSUPPORTED
    assert B.dr_linear_wgrad(q8.handle, p, 128, q, 128, 4, None, w.data_ptr(), 128, 0, None) == B.DR_ERR_UNSUPPORTED
    for bad in (lambda: layer.forward(x[:, :64], None, off), lambda: layer.forward(x, None, off.long()),
                lambda: layer.forward(x.float(), None, off), lambda: layer.wgrad(x, y[:2], off),
                lambda: layer.forward(x, None, off, out=y[:, :64]), lambda: layer.wgrad(x, y, off, accumulate=True),
                lambda: layer.forward(x.t(), None, off), lambda: layer.forward(x.cpu(), None, off)):
        with pytest.raises((ValueError, TypeError)):
            bad()


@pytest.mark.parametrize("fp8", [True, False], ids=["fp8", "bf16"])
def test_offsets_past_32_bits(fp8):
    """Rows that lie more than 2^32 elements behind the first, in x, y and dx."""
    rows, n, k, ld = 70001, 64, 128, 65536
    g = gen(1)
    wide = torch.empty(rows, ld, dtype=torch.uint8 if fp8 else BF16, device=DEV)
    out = torch.empty(rows, ld, dtype=BF16, device=DEV)
    x = torch.randn(rows, k, device=DEV, generator=g)
    w = torch.randn(n, k, device=DEV, generator=g) * 0.05
    if fp8:
        xq, xs = dr.quant_rows(x, wide[:, :k])
        wq, ws = quant_weight(w)
        xd, wd = wide_rows(xq.contiguous().view(torch.float8_e4m3fn), xs), wide_weight(wq, ws)
    else:
        xq, xs, wq, ws = wide[:, :k], None, w.bfloat16(), None
        xq.copy_(x)
        xd, wd = xq.double(), wq.double()
    layer = dr.Linear(wq, ws)
    layer.forward(xq, xs, out=out[:, :n])
    want, tol = product(xd, wd.t(), BF16)
    check(out[:, :n], want, tol)
    if not fp8:
        layer.dgrad(out[:, :n], out=wide[:, 256:256 + k])
        want, tol = product(out[:, :n].double(), wd, BF16)
        check(wide[:, 256:256 + k], want, tol)
        dw = layer.wgrad(xq, out[:, :n])
        want, tol = product(out[:, :n].double().t(), xd, F32)
        check(dw, want, tol)


def test_zz_no_wait_ran_out():
    """After everything above: no kernel gave up waiting for its copies or products."""
    rc, failures = dr.dr_diag_linear_wait_failures()
    assert rc == 0 and failures == 0
