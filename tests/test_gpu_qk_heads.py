"""Norms and rotation of query and key heads: forward, into the cache and back, against 64 bits and against differences."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from attend_util import E4M3, heads, make_cache, scale_above, store
from linear_util import DEV, gen

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
BASE, EPS = 1e6, 1e-6
SHAPES = [(4, 2, 64), (32, 8, 128), (10, 2, 128), (5, 1, 64), (3, 3, 128), (1, 1, 64)]


def unit(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def inputs(seed, rows, n_q, n_kv, dim, dtype, values=True, norms=True):
    g = gen(seed)
    x = (1.7 * torch.randn(rows, (n_q + (2 if values else 1) * n_kv) * dim, device=DEV, generator=g)).to(dtype)
    pos = torch.randint(0, 5000, (rows,), device=DEV, generator=g).int()
    w = [(1 + 0.3 * torch.randn(dim, device=DEV, generator=g)).to(dtype) for _ in range(2)] if norms else [None, None]
    return x, pos, w


def wide(w):
    return [None if t is None else t.double() for t in w]


def tolerance(x, y, pos, n_q, n_kv, dim, w, dtype):
    """fp32 steps: a norm's sum of dim squares (half of (dim + 4) 2^-24 in r), three products, a rotation of two products and a sum of values
    that may each be as large as the pair's; cosines and sines off by 2^-23 and their angle by 2^-32 of a turn: (dim / 2 + 24) 2^-24 of the
    pair's size; then one rounding."""
    size = torch.sqrt(y[..., :dim // 2].square() + y[..., dim // 2:].square()).repeat(1, 1, 2)
    err = (dim / 2 + 24) * 2.0 ** -24 * size
    return err + unit(dtype) * (y.abs() + err) + 1e-40


@pytest.mark.parametrize("n_q,n_kv,dim", SHAPES)
@pytest.mark.parametrize("rows", [1, 7, 300])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norms", [True, False])
def test_forward(n_q, n_kv, dim, rows, dtype, norms):
    x, pos, w = inputs(rows, rows, n_q, n_kv, dim, dtype, norms=norms)
    h = dr.QKHeads(n_q, n_kv, dim, *w, base=BASE, eps=EPS)
    got = h.forward(x, pos)
    want = heads(x.double(), pos, n_q, n_kv, dim, *wide(w), BASE, EPS)
    tol = tolerance(x, want, pos, n_q, n_kv, dim, w, dtype)
    assert ((got.double().view_as(want) - want).abs() <= tol).all()
    same = x.clone()
    h.forward(same, pos, out=same[:, :(n_q + n_kv) * dim])
    assert torch.equal(same[:, :(n_q + n_kv) * dim], got) and torch.equal(same[:, (n_q + n_kv) * dim:], x[:, (n_q + n_kv) * dim:])


@pytest.mark.parametrize("base", [1.0, 10000.0, 5e6])
def test_angles_of_far_positions(base):
    pos = torch.tensor([0, 1, 2, 40960, 131071, 10 ** 6 + 1, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    x, _, _ = inputs(1, len(pos), 4, 2, 128, F32, norms=False)
    got = dr.QKHeads(4, 2, 128, base=base, eps=EPS).forward(x, pos)
    # the definition's own angles in 64 bits are off by 2^-53 * 2^31 radians at the far end, far below the tolerance
    want = heads(x.double(), pos, 4, 2, 128, None, None, base, EPS)
    assert ((got.double().view_as(want) - want).abs() <= tolerance(x, want, pos, 4, 2, 128, None, F32) + 2.0 ** -21).all()


def test_rows_of_negative_position_are_left_as_they_were():
    x, pos, w = inputs(2, 40, 8, 2, 128, BF16)
    pos[::3] = -1
    out = torch.full((40, 10 * 128), 7.0, dtype=BF16, device=DEV)
    h = dr.QKHeads(8, 2, 128, *w)
    h.forward(x, pos, out=out)
    assert (out[::3] == 7).all() and not (out[1::3] == 7).all(1).any()
    dx = torch.full_like(out, 7.0)
    dy = torch.randn(40, 10 * 128, device=DEV, generator=gen(3)).bfloat16()
    _, dq, dk = h.grad(x, pos, dy, dx=dx)
    assert (dx[::3] == 7).all()
    keep = torch.arange(40, device=DEV) % 3 != 0
    _, dq2, dk2 = h.grad(x[keep], pos[keep], dy[keep])
    assert torch.allclose(dq, dq2, rtol=1e-4, atol=1e-4) and torch.allclose(dk, dk2, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(8, 8), (4, 4), (3, 1)])
def test_strides_and_alignments(dtype, pad, shift):
    n_q, n_kv, dim, rows = 6, 2, 64, 33
    x, pos, w = inputs(5, rows, n_q, n_kv, dim, dtype)
    cols, qk = x.shape[1], (n_q + n_kv) * dim
    h = dr.QKHeads(n_q, n_kv, dim, *w)
    want = h.forward(x, pos)
    dy = torch.randn(rows, qk, device=DEV, generator=gen(6)).to(dtype)
    grads = h.grad(x, pos, dy)

    def spread(t):
        buf = torch.full((shift + t.shape[0] * (t.shape[1] + pad),), float("nan"), dtype=t.dtype, device=DEV)
        v = buf[shift:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
        v.copy_(t)
        return v

    assert torch.equal(h.forward(spread(x), pos, out=spread(want.clone().zero_())), want)
    got = h.grad(spread(x), pos, spread(dy), dx=spread(dy.clone().zero_()))
    assert all(torch.equal(a, b) for a, b in zip(got, grads))


def runs_of(rng, lens, starts, block):
    """Runs of requests of `lens` new tokens behind `starts` tokens over scattered blocks, and positions."""
    runs, pos, row, b = [], [], 0, 1
    for n, s in zip(lens, starts):
        at = s
        while at < s + n:
            m = min(block - at % block, s + n - at)
            runs.append([b * 5 % 97, at % block, row, m])
            pos += range(at, at + m)
            at, row, b = at + m, row + m, b + 1
    return runs, pos


@pytest.mark.parametrize("n_q,n_kv,dim", [(4, 2, 64), (32, 8, 128), (5, 1, 64)])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,starts", [([1], [0]), ([1, 1, 1], [5, 15, 127]), ([300, 1, 17, 64], [0, 3, 130, 64])])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_into_the_cache(n_q, n_kv, dim, block, lens, starts, dtype):
    runs, pos = runs_of(None, lens, starts, block)
    rows = sum(lens)
    x, _, w = inputs(rows + block, rows, n_q, n_kv, dim, dtype)
    x[rows // 2] *= 30  # a token that makes a scale grow
    pos = torch.tensor(pos, dtype=torch.int32, device=DEV)
    k, v, ks, vs = make_cache(gen(7), 97, n_kv, block, dim)
    want = [t.double() for t in (k, v, ks, vs)]
    h = dr.QKHeads(n_q, n_kv, dim, *w, base=BASE, eps=EPS)
    cache = dr.KVCache(k, v, ks, vs)
    padded = torch.tensor(runs + [[-1, 0, 0, 0]] * 3, dtype=torch.int32, device=DEV)
    got = h.append(x, pos, padded, cache)
    y = heads(x.double(), pos, n_q, n_kv, dim, *wide(w), BASE, EPS)
    tol = tolerance(x, y, pos, n_q, n_kv, dim, w, dtype)
    assert ((got.double() - y[:, :n_q].reshape(rows, -1)).abs() <= tol[:, :n_q].reshape(rows, -1)).all()
    store(runs, y[:, n_q:], want[0], want[2], block)
    store(runs, x[:, (n_q + n_kv) * dim:].double().view(rows, n_kv, dim), want[1], want[3], block)
    # values come from x itself: their codes and scales are exact; keys' scales are, unless a maximum lies at a border
    assert torch.equal(vs.double(), want[3]) and torch.equal(v.double(), want[1])
    assert torch.equal(ks.double(), want[2])
    # a key within fp32's error of a border between two codes may take either: half a step of the code, and a little
    off, step = (k.double() - want[0]).abs(), torch.exp2(torch.floor(torch.log2(want[0].abs().clamp(min=2.0 ** -6))) - 3)
    assert (off <= step).all() and (off > 0).double().mean() < 1e-3


def test_a_growing_scale_shifts_what_the_block_holds():
    """Token by token or all at once: the values that the block holds are the same but for those below 2^-6 of the last scale."""
    n_q, n_kv, dim, block, rows = 2, 1, 64, 32, 32
    x, _, w = inputs(3, rows, n_q, n_kv, dim, F32)
    x *= torch.exp2(torch.arange(rows, device=DEV)[:, None] * 0.4)
    pos = torch.arange(rows, device=DEV).int()
    h = dr.QKHeads(n_q, n_kv, dim)
    a, b = dr.KVCache.empty(1, n_kv, block, dim), dr.KVCache.empty(1, n_kv, block, dim)
    ints = lambda r: torch.tensor([r], dtype=torch.int32, device=DEV)  # noqa: E731
    h.append(x, pos, ints([0, 0, 0, rows]), a)
    for t in range(rows):
        h.append(x[t:t + 1], pos[t:t + 1], ints([0, t, 0, 1]), b)
    for p, q, ps, qs in ((a.k, b.k, a.k_scale, b.k_scale), (a.v, b.v, a.v_scale, b.v_scale)):
        assert torch.equal(ps, qs)
        u, z = p.double(), q.double()
        big = u.abs() >= 2.0 ** -5
        assert torch.equal(u[big], z[big]) and ((u - z).abs() <= 2.0 ** -9).all()


def test_only_the_runs_slots_are_written():
    n_q, n_kv, dim, block = 4, 2, 64, 32
    x, pos, w = inputs(11, 9, n_q, n_kv, dim, BF16)
    k, v, ks, vs = make_cache(gen(2), 6, n_kv, block, dim, spread=0.0)
    ks.fill_(1.0)
    vs.fill_(1.0)
    before = [t.clone().view(torch.uint8) for t in (k, v)]
    cache = dr.KVCache(k, v, ks, vs)
    dr.QKHeads(n_q, n_kv, dim, *w).append(x, pos, torch.tensor([[2, 7, 0, 9]], dtype=torch.int32, device=DEV), cache)
    for t, b in zip((k, v), before):
        t = t.view(torch.uint8)
        changed = (t != b).any(-1)
        mine = torch.zeros_like(changed)
        mine[2, :, 7:16] = True
        assert not changed[~mine].any() and changed[mine].all()
    assert (ks == 1).all() and (vs == 1).all()


@pytest.mark.parametrize("run", [[-1, 0, 0, 3], [6, 0, 0, 3], [1, -1, 0, 3], [1, 30, 0, 3], [1, 0, 7, 3], [1, 0, -2, 3], [1, 0, 0, 33], [1, 0, 0, -1],
                                 [2 ** 31 - 1, 0, 0, 1], [0, 0, 2 ** 31 - 1, 2]])
def test_runs_that_lie_outside_are_skipped(run):
    n_q, n_kv, dim, block = 4, 2, 64, 32
    x, pos, w = inputs(11, 9, n_q, n_kv, dim, BF16)
    c = dr.KVCache(*make_cache(gen(2), 6, n_kv, block, dim))
    before = [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]
    dr.QKHeads(n_q, n_kv, dim, *w).append(x, pos, torch.tensor([run], dtype=torch.int32, device=DEV), c)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (c.k, c.v, c.k_scale, c.v_scale)))


@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_tokens_that_are_not_finite_are_kept_as_one_nan(where, what):
    n_q, n_kv, dim, block = 4, 2, 64, 16
    x, _, w = inputs(12, 16, n_q, n_kv, dim, BF16)
    pos = torch.arange(16, device=DEV).int()
    h, run = dr.QKHeads(n_q, n_kv, dim, *w), torch.tensor([[0, 0, 0, 16]], dtype=torch.int32, device=DEV)
    a, b = dr.KVCache.empty(1, n_kv, block, dim), dr.KVCache.empty(1, n_kv, block, dim)
    h.append(x, pos, run, a)
    col = (n_q if where == "key" else n_q + n_kv) * dim + dim + 5  # of the second head
    x[9, col] = what
    h.append(x, pos, run, b)
    nan = torch.isnan(b.k.float())
    assert nan[0, 1, 9, 0] and nan.sum() == 1 and not torch.isnan(b.v.float()).any()
    assert torch.isfinite(b.k_scale).all() and torch.isfinite(b.v_scale).all()
    other = torch.arange(16, device=DEV) != 9  # the other tokens are as they were, at whatever scale
    for p, q, ps, qs in ((a.k, b.k, a.k_scale, b.k_scale), (a.v, b.v, a.v_scale, b.v_scale)):
        u, z = p.double() * ps.double()[:, :, None, None], q.double() * qs.double()[:, :, None, None]
        close = (u - z).abs() <= 2.0 ** -9 * torch.maximum(ps, qs).double()[:, :, None, None]
        assert close[:, :, other].all()


@pytest.mark.parametrize("n_q,n_kv,dim", SHAPES)
@pytest.mark.parametrize("rows", [1, 9, 700])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norms", [True, False])
def test_gradients(n_q, n_kv, dim, rows, dtype, norms):
    x, pos, w = inputs(rows + 1, rows, n_q, n_kv, dim, dtype, values=False, norms=norms)
    dy = torch.randn(rows, (n_q + n_kv) * dim, device=DEV, generator=gen(8)).to(dtype)
    h = dr.QKHeads(n_q, n_kv, dim, *w, base=BASE, eps=EPS)
    got = h.grad(x, pos, dy)
    leaves = [x.double().requires_grad_()] + [t.double().requires_grad_() for t in w if t is not None]
    y = heads(leaves[0], pos, n_q, n_kv, dim, *(leaves[1:] if norms else [None, None]), BASE, EPS)
    want = torch.autograd.grad(y, leaves, dy.double().view_as(y))
    # as forward's: some (dim + 40) 2^-24 of |dy| r w and of the mean that is taken off, each at most the head's own size
    size = dy.double().view(rows, n_q + n_kv, dim).norm(dim=-1, keepdim=True)
    xs = x.double().view(rows, n_q + n_kv, dim)
    r = torch.rsqrt(xs.square().mean(-1, keepdim=True) + EPS) if norms else torch.ones_like(size)
    most = max([1.0] + [float(t.abs().max()) for t in w if t is not None])
    err = (dim + 40) * 2.0 ** -24 * size * r * most * (1 + (xs * r).abs() / dim ** 0.5)
    d = want[0].view(rows, n_q + n_kv, dim)
    assert ((got[0].double().view_as(d) - d).abs() <= err + unit(dtype) * (d.abs() + err) + 1e-40).all()
    if not norms:
        assert got[1] is None and got[2] is None
        return
    for g, t, heads_ in ((got[1], want[1], slice(0, n_q)), (got[2], want[2], slice(n_q, None))):
        # products of two fp32 numbers, each off by (dim + 24) 2^-24, summed in fp32 by chains of at most rows * heads
        mass = (dy.double().view(rows, -1, dim)[:, heads_].norm(dim=-1, keepdim=True) * (xs * r)[:, heads_].abs()).sum((0, 1))
        count = xs[:, heads_].shape[1] * rows
        assert ((g.double() - t).abs() <= (dim + 24 + count) * 2.0 ** -24 * mass + 1e-30).all()
    base = [t.clone() for t in got[1:]]
    again = h.grad(x, pos, dy, dx=dy.clone(), dq_norm=base[0], dk_norm=base[1], accumulate=True)
    assert torch.equal(again[1], got[1] + got[1]) and torch.equal(again[2], got[2] + got[2])
    same = dy.clone()
    h.grad(x, pos, same, dx=same)
    assert torch.equal(same, got[0])


def test_gradients_against_differences():
    n_q, n_kv, dim, rows = 2, 1, 64, 3
    x, pos, w = inputs(21, rows, n_q, n_kv, dim, F32, values=False)
    pos = pos % 50
    dy = torch.randn(rows, (n_q + n_kv) * dim, device=DEV, generator=gen(9))
    dx, dq, dk = dr.QKHeads(n_q, n_kv, dim, *w, base=BASE, eps=EPS).grad(x, pos, dy)
    xs, ws = x.double(), wide(w)

    def loss(x_, w_):
        return float((heads(x_, pos, n_q, n_kv, dim, *w_, BASE, EPS).reshape(rows, -1) * dy.double()).sum())

    step = 2.0 ** -16  # differences of the 64-bit form: off by step^2 times a third derivative, and 2^-53 / step
    for where in [(0, 0), (1, 37), (2, 130), (0, 191)]:
        d = torch.zeros_like(xs)
        d[where] = step
        num = (loss(xs + d, ws) - loss(xs - d, ws)) / (2 * step)
        assert abs(num - float(dx[where])) <= 1e-4 * float(dy.norm())
    for g, i in ((dq, 0), (dk, 1)):
        for at in (0, 31, 63):
            up, down = [t.clone() for t in ws], [t.clone() for t in ws]
            up[i][at] += step
            down[i][at] -= step
            assert abs((loss(xs, up) - loss(xs, down)) / (2 * step) - float(g[at])) <= 1e-4 * float(dy.norm())


def test_no_rows():
    h = dr.QKHeads(4, 2, 64, *[torch.ones(64, device=DEV)] * 2)
    x, pos = torch.empty(0, 6 * 64, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    assert h.forward(x, pos).shape == (0, 6 * 64)
    dq = torch.full((64,), 5.0, device=DEV)
    _, dq, dk = h.grad(x, pos, x, dq_norm=dq)
    assert (dq == 0).all() and (dk == 0).all()
    _, dq, dk = h.grad(x, pos, x, dq_norm=dq.fill_(5), dk_norm=dk.fill_(5), accumulate=True)
    assert (dq == 5).all() and (dk == 5).all()


def test_captured_and_replayed():
    x, pos, w = inputs(31, 500, 8, 2, 128, BF16)
    dy = torch.randn(500, 10 * 128, device=DEV, generator=gen(10)).bfloat16()
    h = dr.QKHeads(8, 2, 128, *w)
    want, grads = h.forward(x, pos), h.grad(x, pos, dy)
    y, dx, dq, dk = torch.zeros_like(want), torch.zeros_like(dy), torch.zeros(128, device=DEV), torch.zeros(128, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.forward(x, pos, out=y)
        h.grad(x, pos, dy, dx=dx, dq_norm=dq, dk_norm=dk)
    for _ in range(2):
        for t in (y, dx, dq, dk):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, grads[0]) and torch.equal(dq, grads[1]) and torch.equal(dk, grads[2])
