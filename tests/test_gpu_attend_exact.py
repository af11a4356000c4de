"""Attention whose logits are whole numbers times a power of two: sums of products are exact, so that little but p and the output is rounded."""
import math

import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen

pytestmark = pytest.mark.gpu
DIM, BLOCK, N_Q, KV, SCALE = 128, 32, 8, 2, 2.0 ** -5


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def case(seed, n, rows, common, climb):
    """Whole numbers: half of the dimensions give every token a logit near `common`, with climb > 0 rising by climb from block to block, the
    others differences of some units.  Products of a logit sum to less than 2^24."""
    g = gen(seed)
    blocks = -(-n // BLOCK)
    draw = lambda lo, hi, *shape: torch.randint(lo, hi, shape, device=DEV, generator=g).float()  # noqa: E731
    q = torch.cat([draw(129, 256, rows, N_Q, 64), draw(17, 32, rows, N_Q, 64) * (2 * draw(0, 2, rows, N_Q, 64) - 1)], -1)
    k = torch.cat([torch.zeros(blocks, KV, BLOCK, 64, device=DEV), draw(-1, 2, blocks, KV, BLOCK, 64)], -1)
    # 64 dimensions times about 192: each code of 1 there adds 384 to the logit of every row, give or take some
    k[..., :64] = round(common / (64 * 192 * SCALE))
    assert float(k[..., 0].max()) in (0, 1, 5, 64)  # codes hold these exactly
    if climb:
        for b in range(blocks):
            k[b, :, :, 0] += [0, 1, 2, 4, 6, 8, 10, 12, 14, 16][b % 10] * climb
    v = torch.randn(blocks, KV, BLOCK, DIM, device=DEV, generator=g).to(torch.float8_e4m3fn)
    order = torch.randperm(blocks, device=DEV, generator=g)
    table = torch.empty(1, blocks, dtype=torch.int32, device=DEV)
    table[0, :] = order.int()
    kk = torch.empty_like(k)
    kk[order] = k  # block j of the request lies in block order[j] of the cache
    codes = kk.to(torch.float8_e4m3fn)
    assert torch.equal(codes.float(), kk)
    return q.view(rows, -1).bfloat16(), codes, v, table


def plain(q, codes, v, table, n, rows):
    """(out, allowed error) in 64 bits.  log2 of p is a whole number times a factor, both exact or rounded once or twice, in one addition, less a maximum:
    off by 2^-22 of itself and of the row's largest; p by that, by 2^-11 (fp16), 2^-18 (exponential), 2^-36 of the largest; the sums of n by
    (n + 8) 2^-23, the result by 2^-8.  Each token's error counts by its p."""
    out, tol = [], []
    ids = table[0].long()
    t, pos = torch.arange(n, device=DEV)[None], torch.arange(n - rows, n, device=DEV)[:, None]
    for h in range(N_Q):
        c = h // (N_Q // KV)
        kk, vv = (x[ids, c].double().reshape(-1, DIM)[:n] for x in (codes, v))
        dots = q[:, h * DIM:(h + 1) * DIM].double() @ kk.t()
        assert float(dots.abs().max()) < 2 ** 24
        s = torch.where(t <= pos, SCALE * dots, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.softmax(s, 1)
        off = 2.0 ** -22 * torch.where(t <= pos, s.abs() + top.abs(), 0.0)
        off = torch.expm1(off) + 2.0 ** -11 + 2.0 ** -18 + (n + 8) * 2.0 ** -23
        y = p @ vv
        err = (p * off) @ vv.abs() + y.abs() * (p * off).sum(1, keepdim=True) + 2.0 ** -36 * p.amax(1, keepdim=True) * ((t <= pos).double() @ vv.abs())
        err = err + 2.0 ** -12 * err  # second order
        out.append(y)
        tol.append(err + 2.0 ** -8 * (y.abs() + err))
    return torch.cat(out, 1), torch.cat(tol, 1)


@pytest.mark.parametrize("rows", [1, 5, 15, 40, 150])
@pytest.mark.parametrize("common,climb", [(0, 0), (384, 0), (2000, 0), (24576, 0), (0, 1), (0, 4)])
def test_large_logits(rows, common, climb):
    n = 400
    q, codes, v, table = case(rows + common, n, rows, common, climb)
    ones = torch.ones(codes.shape[:2], device=DEV)
    cache = dr.KVCache(codes, v, ones, ones.clone())
    got = cache.attend(q, ints([n]), table, ints([0, rows]), scale=SCALE).double()
    want, tol = plain(q, codes, v, table, n, rows)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {float(((got - want).abs() / tol).max())} times what is allowed"
    # what this does not take: nothing, queries of the other sign, queries of four significant bits
    e = torch.floor(torch.log2(q.float().abs()))
    short = (torch.round(q.float() / torch.exp2(e - 3)) * torch.exp2(e - 3)).bfloat16()
    for wrong in (torch.zeros_like(want), plain(-q, codes, v, table, n, rows)[0], plain(short, codes, v, table, n, rows)[0]):
        assert ((wrong - want).abs() > tol).double().mean() > 0.3
