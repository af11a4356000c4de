"""Attention over the 8-bit cache against 64 bits: heads, lengths, block sizes, windows, rows that see nothing, garbage in masked places."""
import itertools

import pytest
import torch

import paper_2607_22614_b200 as dr
from attend_util import E4M3, attention, make_cache, make_table
from linear_util import DEV, gen

pytestmark = pytest.mark.gpu


def setup(seed, lengths, added, n_q, kv, dim, block, garbage=True, spare=3, queries=1.5):
    g = gen(seed)
    n_blocks = sum(-(-n // block) for n in lengths) + spare
    k, v, ks, vs = make_cache(g, n_blocks, kv, block, dim)
    width = max(-(-n // block) for n in lengths) + 2
    table = make_table(g, lengths, block, n_blocks, width)
    if garbage:  # slots behind a request's last token hold NaN codes, blocks that nobody has hold them too
        owned = torch.zeros(n_blocks, block, dtype=torch.bool, device=DEV)
        for r, n in enumerate(lengths):
            for j in range(-(-n // block)):
                owned[int(table[r, j]), :min(block, n - j * block)] = True
        for c in (k, v):
            c.view(torch.uint8).masked_fill_(~owned[:, None, :, None], 0x7F)
    offsets = [0]
    for a in added:
        offsets.append(offsets[-1] + a)
    q = (queries * torch.randn(offsets[-1], n_q * dim, device=DEV, generator=g)).bfloat16()
    return q, (k, v, ks, vs), table, offsets


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def check(q, cache, table, lengths, offsets, n_q, window=0, sinks=0, scale=None, use_offsets=True, out=None):
    c = dr.KVCache(*cache)
    got = c.attend(q, ints(lengths), table, ints(offsets) if use_offsets else None, window=window, sinks=sinks, scale=scale, out=out)
    want, tol = attention(q, *cache, lengths, offsets, table, n_q, window, sinks, scale)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, first {bad.nonzero()[0].tolist()}: " \
        f"{got[tuple(bad.nonzero()[0])].item()} for {want[tuple(bad.nonzero()[0])].item()} (allowed {tol[tuple(bad.nonzero()[0])].item()})"
    rc, failed = dr.dr_diag_linear_wait_failures()
    assert rc == 0 and failed == 0
    return got


HEADS = [(4, 2, 64), (8, 8, 128), (32, 8, 128), (10, 2, 128), (8, 1, 128), (16, 1, 64), (48, 2, 128)]


@pytest.mark.parametrize("n_q,kv,dim", HEADS)
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_one_token(n_q, kv, dim, block):
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 129, 500, 1023]
    q, cache, table, offsets = setup(n_q + block, lengths, [1] * len(lengths), n_q, kv, dim, block)
    check(q, cache, table, lengths, offsets, n_q, use_offsets=False)


@pytest.mark.parametrize("lengths", [[1], [4000], [20000, 3], [3, 0, 700, 0], [0]])
def test_few_and_many_parts(lengths):
    q, cache, table, offsets = setup(len(lengths), lengths, [1] * len(lengths), 8, 2, 128, 64)
    got = check(q, cache, table, lengths, offsets, 8, use_offsets=False)
    for r, n in enumerate(lengths):
        if n == 0:
            assert (got[r] == 0).all()


@pytest.mark.parametrize("n_q,kv,dim", [(32, 8, 128), (10, 2, 128), (4, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("added", [[2, 5, 1, 8, 0, 3], [17, 33, 1, 64, 0, 7], [200, 1, 129, 0, 300, 5]])
@pytest.mark.parametrize("block", [16, 128])
def test_several_tokens(n_q, kv, dim, added, block):
    lengths = [max(a, n) for a, n in zip(added, [2, 700, 1, 130, 40, 333])]
    q, cache, table, offsets = setup(sum(added) + block, lengths, added, n_q, kv, dim, block)
    check(q, cache, table, lengths, offsets, n_q)


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (64, 4), (100, 1), (100, 70), (5000, 4), (130, 129), (1 << 40, 3)])
@pytest.mark.parametrize("added", [[1, 1, 1, 1], [3, 8, 1, 2], [150, 260, 1, 90]])
def test_windows_and_sinks(window, sinks, added):
    lengths = [max(a, n) for a, n in zip(added, [5, 1000, 131, 90])]
    q, cache, table, offsets = setup(window % 1000 + sinks, lengths, added, 8, 2, 128, 32)
    check(q, cache, table, lengths, offsets, 8, min(window, 1 << 30), sinks)


@pytest.mark.parametrize("added", [[1, 1], [4, 3], [200, 130]])
def test_blocks_that_are_not_held_are_hidden(added):
    """Entries outside the cache stand for blocks that have been given back, say behind a window."""
    lengths = [500, 260]
    q, cache, table, offsets = setup(5, lengths, added, 8, 2, 128, 32)
    table[0, 2:6] = -1
    table[0, 9] = cache[0].shape[0]
    table[1, 0] = 2 ** 31 - 1
    check(q, cache, table, lengths, offsets, 8)
    table[1, :] = -1  # nothing is left to see
    got = check(q, cache, table, lengths, offsets, 8)
    assert (got[offsets[1]:offsets[2]] == 0).all()


@pytest.mark.parametrize("n,a", [(3, 5), (0, 2), (100, 160)])
def test_rows_before_the_first_token_see_nothing(n, a):
    lengths, added = [n, 70], [a, 1]
    q, cache, table, offsets = setup(9, lengths, added, 8, 2, 128, 32)
    got = check(q, cache, table, lengths, offsets, 8)
    assert (got[:a - n] == 0).all()


@pytest.mark.parametrize("added", [[1, 1, 1], [5, 3, 6], [140, 1, 40]])
def test_strides_alignments_and_rows_that_nobody_owns(added):
    lengths = [300, 41, 77]
    q, cache, table, offsets = setup(11, lengths, added, 6, 2, 64, 16)
    rows, cols = q.shape
    want = check(q, cache, table, lengths, offsets, 6)
    for pad, shift in ((8, 0), (64, 4), (3, 1), (5, 2)):
        buf = torch.full((shift + (rows + 2) * (cols + pad),), float("nan"), dtype=torch.bfloat16, device=DEV)
        wide = buf[shift:].view(rows + 2, cols + pad)[:, :cols]
        wide[:rows] = q
        out = torch.full((shift + (rows + 2) * (cols + pad),), 7.0, dtype=torch.bfloat16, device=DEV)
        to = out[shift:].view(rows + 2, cols + pad)
        padded = torch.full((3, table.shape[1] + 5), -1, dtype=torch.int32, device=DEV)
        padded[:, :table.shape[1]] = table
        dr.KVCache(*cache).attend(wide, ints(lengths), padded[:, :table.shape[1]], ints(offsets), out=to[:, :cols])
        assert torch.equal(to[:rows, :cols], want)
        assert (to[rows:] == 7).all() and (to[:, cols:] == 7).all() and (out[:shift] == 7).all()


@pytest.mark.parametrize("added", [[1, 1], [3, 2], [130, 64]])
@pytest.mark.parametrize("queries", [1e-30, 40.0, 1e4])
def test_small_and_large_logits(added, queries):
    lengths = [400, 130]
    q, cache, table, offsets = setup(13, lengths, added, 8, 2, 128, 32, queries=queries)
    check(q, cache, table, lengths, offsets, 8)


@pytest.mark.parametrize("added", [[1, 1], [130, 64]])
def test_scale_and_blocks_of_very_different_sizes(added):
    lengths = [400, 130]
    q, cache, table, offsets = setup(13, lengths, added, 8, 2, 128, 32)
    k, v, ks, vs = cache
    vs *= torch.exp2(torch.randint(-60, 60, vs.shape, device=DEV, generator=gen(1)).float())
    ks[::3] = 2.0 ** -100
    check(q, cache, table, lengths, offsets, 8, scale=0.3)
    check(q, cache, table, lengths, offsets, 8, scale=-0.1)
    vs[int(table[0, 0])] = 2.0 ** -100
    v[int(table[0, 0])] = torch.zeros_like(v[int(table[0, 0])])
    check(q, cache, table, lengths, offsets, 8)


@pytest.mark.parametrize("added", [[1, 1, 1], [6, 2, 1], [140, 90, 1]])
def test_poisoned_tokens_reach_only_the_rows_that_see_them(added):
    """A NaN key makes the rows that see it NaN, and no others."""
    lengths = [300, 100, 7]
    q, cache, table, offsets = setup(17, lengths, added, 8, 2, 128, 32)
    k = cache[0]
    bad = lengths[0] - added[0] // 2 - 1
    k[int(table[0, bad // 32]), 1, bad % 32, 0] = float("nan")
    got = dr.KVCache(*cache).attend(q, ints(lengths), table, ints(offsets))
    want, tol = attention(q, *cache, lengths, offsets, table, 8)
    nan = torch.zeros_like(want, dtype=torch.bool)
    first = bad - (lengths[0] - added[0])
    nan[max(first, 0):added[0], 4 * 128:] = True
    assert torch.equal(torch.isnan(got), nan)
    assert ((got.double() - want).abs() <= tol)[~nan].all()


@pytest.mark.parametrize("added", [[1] * 9, [4] * 9, [70] * 9])
def test_the_same_call_gives_the_same_bits_on_every_stream_and_replayed(added):
    lengths = [1000 + 37 * i for i in range(9)]
    q, cache, table, offsets = setup(19, lengths, added, 8, 2, 128, 64)
    c, L, o = dr.KVCache(*cache), ints(lengths), ints(offsets)
    want = c.attend(q, L, table, o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [c.attend(q, L, table, o, stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in outs)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.graph(graph):
        c.attend(q, L, table, o, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    # lengths are read at each replay
    L -= 64
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, c.attend(q, L, table, o))
    rc, failed = dr.dr_diag_linear_wait_failures()
    assert rc == 0 and failed == 0


def test_many_requests():
    lengths = [(i * 37) % 200 for i in range(700)]
    q, cache, table, offsets = setup(23, lengths, [1] * 700, 4, 2, 64, 32)
    check(q, cache, table, lengths, offsets, 4, use_offsets=False)


def test_lengths_and_offsets_out_of_range_stay_inside():
    q, cache, table, offsets = setup(29, [100, 60], [1, 1], 8, 2, 128, 32)
    c = dr.KVCache(*cache)
    for lengths, off in (([2 ** 31 - 1, 60], [0, 1, 2]), ([-5, 60], [0, 1, 2]), ([100, 60], [-4, 1, 900]), ([100, 60], [2, 1, 0])):
        c.attend(q, ints(lengths), table, ints(off))
    torch.cuda.synchronize()
    rc, failed = dr.dr_diag_linear_wait_failures()
    assert rc == 0 and failed == 0


@pytest.mark.parametrize("added", [[1, 1], [6, 2], [140, 90]])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_query_rows_that_are_not_finite_give_nan_and_spoil_no_others(added, what):
    lengths = [300, 100]
    q, cache, table, offsets = setup(31, lengths, added, 8, 2, 128, 32)
    want = dr.KVCache(*cache).attend(q, ints(lengths), table, ints(offsets))
    bad = added[0] // 2
    q[bad, 5 * 128 + 17] = what
    got = dr.KVCache(*cache).attend(q, ints(lengths), table, ints(offsets))
    nan = torch.zeros_like(want, dtype=torch.bool)
    nan[bad, 5 * 128:6 * 128] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("added", [[1, 1], [70, 3]])
def test_codes_as_bytes_and_a_table_that_shares_blocks(added):
    """uint8 codes are e4m3 codes; two requests may share the blocks of a common prefix."""
    lengths = [200, 170]
    q, cache, table, offsets = setup(37, lengths, added, 8, 2, 64, 32, garbage=False)
    table[1, :3] = table[0, :3]
    want = check(q, cache, table, lengths, offsets, 8)
    k, v, ks, vs = cache
    got = dr.KVCache(k.view(torch.uint8), v.view(torch.uint8), ks, vs).attend(q, ints(lengths), table, ints(offsets))
    assert torch.equal(got, want)


@pytest.mark.parametrize("added", [[1], [90]])
def test_a_cache_beyond_four_gigabytes(added):
    """Blocks whose codes lie past 2^32 bytes, written by append and read by attend."""
    n_blocks, kv, block, dim, n = 300000, 2, 64, 128, 150
    assert n_blocks * kv * block * dim > 1 << 32
    c = dr.KVCache.empty(n_blocks, kv, block, dim)
    table = ints([[n_blocks - 1, n_blocks - 7, 3]])
    heads = dr.QKHeads(8, kv, dim)
    x = torch.randn(n, 12 * dim, device=DEV, generator=gen(41)).bfloat16()
    runs = ints([[n_blocks - 1, 0, 0, 64], [n_blocks - 7, 0, 64, 64], [3, 0, 128, 22]])
    q = heads.append(x, torch.arange(n, device=DEV).int(), runs, c)[n - added[0]:]
    got = c.attend(q, ints([n]), table, ints([0, added[0]]))
    held = table[0].long()
    near = torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEV)
    want, tol = attention(q, c.k[held], c.v[held], c.k_scale[held], c.v_scale[held], [n], [0, added[0]], near, 8)
    assert ((got.double() - want).abs() <= tol).all()
