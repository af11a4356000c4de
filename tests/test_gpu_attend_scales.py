"""Attention over blocks whose value scales lie far apart: blocks without values, which append gives the scale 2^-100, beside large ones."""
import math

import pytest
import torch

import paper_2607_22614_b200 as dr
from attend_util import attention, make_cache, make_table
from linear_util import DEV, gen

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -100
N_Q, KV, DIM = 8, 2, 128


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def setup(seed, lengths, added, block, dim=DIM):
    """Queries, a cache whose keys and values are normal, a table, offsets."""
    g = gen(seed)
    n_blocks = sum(-(-n // block) for n in lengths) + 3
    cache = make_cache(g, n_blocks, KV, block, dim, spread=0.0)
    table = make_table(g, lengths, block, n_blocks, max(-(-n // block) for n in lengths) + 2)
    offsets = [sum(added[:i]) for i in range(len(added) + 1)]
    return (1.5 * torch.randn(offsets[-1], N_Q * dim, device=DEV, generator=g)).bfloat16(), cache, table, offsets


def below_fp16(q, k, v, k_scale, v_scale, lengths, offsets, table, window, sinks):
    """p times a block's scale is rounded to fp16 relative to the row's largest such product, which is at least 2^11: below 2^-14 that is
    half a step of 2^-24, 2^-36 of the largest for each code."""
    block, dim = k.shape[2:]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for r, n in enumerate(lengths):
        lo, hi = offsets[r], offsets[r + 1]
        ids = table[r, :-(-n // block)].long()
        pos, t = torch.arange(n - (hi - lo), n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
        seen = t <= pos
        if window:
            seen &= (t > pos - window) | (t < sinks)
        for h in range(N_Q):
            c = h // (N_Q // KV)
            kk = (k[ids, c].double() * k_scale[ids, c].double()[:, None, None]).reshape(-1, dim)[:n]
            codes = v[ids, c].double().abs().reshape(-1, dim)[:n]
            s = torch.where(seen, dim ** -0.5 * (q[lo:hi, h * dim:(h + 1) * dim].double() @ kk.t()), -math.inf)
            most = (torch.softmax(s, 1) * v_scale[ids, c].double().repeat_interleave(block)[:n]).amax(1, keepdim=True)
            out[lo:hi, h * dim:(h + 1) * dim] = 2.0 ** -36 * most * (seen.double() @ codes)
    return out


def check(q, cache, table, lengths, offsets, window=0, sinks=0):
    got = dr.KVCache(*cache).attend(q, ints(lengths), table, ints(offsets), window=window, sinks=sinks)
    want, tol = attention(q, *cache, lengths, offsets, table, N_Q, window, sinks)
    tol += below_fp16(q, *cache, lengths, offsets, table, window, sinks)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, first {bad.nonzero()[0].tolist()}: " \
        f"{got[tuple(bad.nonzero()[0])].item()} for {want[tuple(bad.nonzero()[0])].item()} (allowed {tol[tuple(bad.nonzero()[0])].item()})"


def without_values(cache, ids):
    _, v, _, vs = cache
    v[ids] = torch.zeros_like(v[ids])
    vs[ids] = LEAST


@pytest.mark.parametrize("added", [[1, 1], [9, 3], [40, 17], [150, 80]])
@pytest.mark.parametrize("top", [-110, -60, 20, 36, 40, 90, 110])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("first", [0, 1])
def test_every_other_block_has_no_values(added, top, block, first):
    """Visible ones belong to the sum of p as any other block does; those that a row does not see yet add nothing to it."""
    lengths = [333, 170]
    q, cache, table, offsets = setup(block, lengths, added, block)
    cache[3].fill_(2.0 ** top)
    for r, n in enumerate(lengths):
        without_values(cache, table[r, first:-(-n // block):2].long())
    check(q, cache, table, lengths, offsets)
    check(q, cache, table, lengths, offsets, window=100, sinks=20)


@pytest.mark.parametrize("added", [[1, 1], [9, 3], [150, 80]])
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_over_their_whole_range(added, dim):
    lengths = [700, 170]
    q, cache, table, offsets = setup(3, lengths, added, 16, dim)
    for seed in range(4):
        cache[3].copy_(torch.exp2(torch.randint(-126, 118, cache[3].shape, device=DEV, generator=gen(seed)).float()))
        check(q, cache, table, lengths, offsets)


@pytest.mark.parametrize("rows", [1, 3, 6, 14])
def test_parts_of_many_groups(rows):
    """Groups of eight, sixteen and 24 rows of which several CTAs have parts, some with sums of their own and some without."""
    lengths = [600 + 17 * i for i in range(60)]
    added = [rows] * 60
    q, cache, table, offsets = setup(11, lengths, added, 32)
    for r in range(60):
        if r % 3:
            without_values(cache, table[r, r % 7:-(-lengths[r] // 32):1 + r % 5].long())
    cache[3][table[::4, 2].long()] = 2.0 ** 60
    check(q, cache, table, lengths, offsets)
    check(q, cache, table, lengths, offsets, window=300, sinks=40)


@pytest.mark.parametrize("added", [[1], [6], [150]])
def test_scales_that_are_no_powers_of_two(added):
    q, cache, table, offsets = setup(4, [400], added, 32)
    cache[3].mul_(1 + torch.rand(cache[3].shape, device=DEV, generator=gen(5)))
    check(q, cache, table, [400], offsets)
    cache[3][::2] *= 2.0 ** 60
    check(q, cache, table, [400], offsets)


@pytest.mark.parametrize("added", [1, 5, 40])
def test_a_long_context_without_values(added):
    """Tens of thousands of tokens whose values are zero, each p up to 2^4 times the first one's, before one block that has values."""
    n, block = 60000, 64
    q, cache, table, offsets = setup(6, [n], [added], block)
    k, v, ks, vs = cache
    q.fill_(1.0)
    k.copy_(torch.full(k.shape, 2.0, device=DEV).to(k.dtype))
    ks.fill_(3.8 / 1.4426950408889634 * DIM ** 0.5 / (2 * DIM))  # every logit 3.8 / log2(e)
    ids = table[0, :-(-n // block)].long()
    k[ids[0]] = torch.zeros_like(k[ids[0]])                       # but the first block's: 0
    held = ids[(n - added - 200) // block]
    kept = v[held].clone(), vs[held].clone()
    without_values(cache, ids)
    v[held], vs[held] = kept
    check(q, cache, table, [n], offsets)


@pytest.mark.parametrize("added", [1, 5, 40])
def test_a_token_that_sees_itself_alone_gets_its_values(added):
    """Of each size that values may have, rounded once."""
    for e in (-126, -119, -100, -41, -40, 0, 40, 41, 100, 118):
        q, cache, table, offsets = setup(e + 200, [added], [added], 16)
        cache[3].fill_(2.0 ** e)
        got = dr.KVCache(*cache).attend(q, ints([added]), table, ints(offsets))
        want = (cache[1][int(table[0, 0]), :, 0].double() * 2.0 ** e).repeat_interleave(N_Q // KV, 0).reshape(-1)
        # (a step of bf16 is 2^-133 at least)
        assert ((got[0].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -18) * want.abs() + 2.0 ** -134).all(), e


@pytest.mark.parametrize("added", [[1, 1], [9, 3], [150, 80]])
@pytest.mark.parametrize("what", ["query", "key"])
def test_rows_that_are_not_finite_spoil_no_others(added, what):
    lengths = [333, 170]
    q, cache, table, offsets = setup(7, lengths, added, 16)
    cache[3].mul_(torch.exp2(torch.randint(-90, 90, cache[3].shape, device=DEV, generator=gen(8)).float()))
    without_values(cache, table[0, 3:20:4].long())
    c, L, O = dr.KVCache(*cache), ints(lengths), ints(offsets)
    want = c.attend(q, L, table, O)
    nan = torch.zeros_like(want, dtype=torch.bool)
    if what == "query":
        q[added[0] // 2, 5 * DIM + 17] = math.inf
        nan[added[0] // 2, 5 * DIM:6 * DIM] = True
    else:  # a token among the first request's new ones, in a block without values
        at = lengths[0] - 1 - added[0] // 2
        without_values(cache, table[0, at // 16:at // 16 + 1].long())
        want = c.attend(q, L, table, O)
        cache[0][int(table[0, at // 16]), 1, at % 16, 0] = math.nan
        nan[added[0] - 1 - added[0] // 2:added[0], 4 * DIM:] = True
    got = c.attend(q, L, table, O)
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
    assert torch.isfinite(want).all()


@pytest.mark.parametrize("added", [[1, 1], [9, 3], [150, 80]])
def test_a_scale_of_zero_is_a_block_without_values(added):
    lengths = [333, 170]
    q, cache, table, offsets = setup(9, lengths, added, 16)
    cache[3][table[0, 2:18:5].long()] = 0.0
    check(q, cache, table, lengths, offsets)
