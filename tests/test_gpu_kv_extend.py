"""Block tables, positions and runs of slots against plain Python."""
import random

import pytest
import torch

import paper_2607_22614_b200 as dr
from attend_util import extend

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def cache(n_blocks, block):
    return dr.KVCache.empty(n_blocks, 1, block, 64)


def state_of(rng, requests, block, width, longest, spare):
    """Lengths, a table over scattered blocks, a free list of the others."""
    lengths = [min(rng.randint(0, longest), width * block) for _ in range(requests)]
    need = [-(-n // block) for n in lengths]
    ids = list(range(sum(need) + spare))
    rng.shuffle(ids)
    table, at = [], 0
    for n in need:
        table.append(ids[at:at + n] + [-9] * (width - n))
        at += n
    return lengths, table, ids[at:] + [-9] * at, [spare, 77], len(ids)


def check(c, added, lengths, table, free, state, rows, in_place, pad=0):
    R, W = len(lengths), len(table[0])
    n_runs = c.runs_for(R, rows)
    want = extend(added, lengths, table, free, state, rows, c.block_tokens, c.n_blocks, n_runs)
    T = torch.full((R, W + pad), -3, dtype=torch.int32, device=DEV)
    T[:, :W] = ints(table)
    L, F, S = ints(lengths), ints(free), ints(state)
    kw = {} if in_place else dict(lengths_out=torch.empty_like(L), state_out=torch.empty_like(S))
    offsets, positions, runs = c.extend(ints(added), L, T[:, :W], F, S, rows, **kw)
    got = (offsets, positions, runs, L if in_place else kw["lengths_out"], T[:, :W], F, S if in_place else kw["state_out"])
    count = want[6][0]
    for name, g, w in zip(("offsets", "positions", "runs", "lengths", "table", "free", "state"), got, want):
        g = g.tolist()
        if name == "free":  # what the list holds behind its end is of no account
            g, w = g[:count], w[:count]
        assert g == w, f"{name}: {[(i, a, b) for i, (a, b) in enumerate(zip(g, w)) if a != b][:4]}"
    assert (T[:, W:] == -3).all()
    if not in_place:
        assert L.tolist() == list(lengths) and S.tolist() == list(state)
    return offsets, positions, runs, L, T, F, S


@pytest.mark.parametrize("requests", [1, 3, 64, 511, 513, 1500])
@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("kind", ["decode", "mixed", "prompts"])
@pytest.mark.parametrize("in_place", [True, False])
def test_steps(requests, block, kind, in_place):
    rng = random.Random(requests * 7 + block)
    width = 24
    lengths, table, free, state, n = state_of(rng, requests, block, width, width * block // 2, requests * 6 + 3)
    if kind == "decode":
        added = [1] * requests
    elif kind == "mixed":
        added = [rng.choice([-1, 0, 1, 1, 2, block, rng.randint(1, 3 * block)]) for _ in range(requests)]
    else:
        added = [rng.randint(1, 5 * block) for _ in range(requests)]
    c = cache(n, block)
    rows = sum(max(a, 0) for a in added)
    check(c, added, lengths, table, free, state, rows, in_place, pad=3)
    check(c, added, lengths, table, free, state, rows + 50, in_place)


@pytest.mark.parametrize("requests", [5, 600])
@pytest.mark.parametrize("lack", ["blocks", "rows", "width", "none left"])
def test_refused_requests(requests, lack):
    rng = random.Random(requests)
    block, width = 32, 8
    lengths, table, free, state, n = state_of(rng, requests, block, width, 100, requests * 3)
    added = [rng.randint(0, 90) for _ in range(requests)]
    rows = sum(added)
    if lack == "blocks":
        state = [requests // 2, 0]
    elif lack == "none left":
        state = [0, 0]
    elif lack == "rows":
        rows = rows * 2 // 3
    else:
        added = [rng.choice([5, 400, 1]) for _ in range(requests)]
        rows = sum(added)
    check(cache(n, block), added, lengths, table, free, state, rows, False)


def test_blocks_that_come_back_are_taken_at_once():
    block = 16
    lengths, table, free, state = [40, 20, 0, 33], [[4, 5, 6, -1], [7, 8, -1, -1], [-1] * 4, [0, 1, 2, -1]], [3] + [-9] * 8, [1, 0]
    got = check(cache(9, block), [-1, 13, 50, -1], lengths, table, free, state, 63, True)
    assert got[3].tolist() == [0, 33, 50, 0] and got[6].tolist() == [2, 0]


def test_a_sequence_from_start_to_end_loses_no_block():
    rng = random.Random(4)
    block, n, R, W = 16, 60, 7, 20
    c = cache(n, block)
    lengths, table, free, state = [0] * R, [[-1] * W for _ in range(R)], list(range(n)), [n, 0]
    L, T, F, S = ints(lengths), ints(table), ints(free), ints(state)
    for step in range(40):
        added = [rng.choice([-1, 0, 1, 1, 1, 20, 60]) for _ in range(R)]
        rows = sum(max(a, 0) for a in added)
        w = extend(added, L.tolist(), T.tolist(), F.tolist(), S.tolist(), rows, block, n, c.runs_for(R, rows))
        o, p, r = c.extend(ints(added), L, T, F, S, rows)
        assert [x.tolist() for x in (o, p, r, L, T, S)] == [w[0], w[1], w[2], w[3], w[4], w[6]], step
        mine = [b for i in range(R) for b in T[i, :-(-int(L[i]) // block)].tolist()]
        assert sorted(mine + F[:int(S[0])].tolist()) == list(range(n)), step


def test_nothing_to_do():
    c = cache(4, 16)
    check(c, [0, 0], [3, 0], [[1], [-1]], [0, 2, 3, -1], [3, 0], 0, True)
    check(c, [0, -1], [3, 0], [[1], [-1]], [0, 2, 3, -1], [3, 0], 5, True)


def test_values_out_of_range_stay_inside():
    c = cache(4, 16)
    check(c, [5, 2 ** 31 - 1, -2 ** 31, 3], [2 ** 31 - 1, 0, -4, 1], [[1, 2]] * 4, [0, 2, 3, -1], [99, 0], 20, False)
    check(c, [2 ** 31 - 1] * 3, [0, 0, 0], [[1, 2]] * 3, [0, 2, 3, -1], [-8, 0], 20, False)


def test_replayed_steps():
    """A decode step captured once: every replay moves the requests on by one token."""
    block, n, R, W = 16, 40, 5, 10
    c = cache(n, block)
    lengths, table, free, state = [3, 15, 16, 0, 31], [[-1] * W for _ in range(R)], list(range(n)), [n, 0]
    for r, m in enumerate(lengths):
        for j in range(-(-m // block)):
            state[0] -= 1
            table[r][j] = free[state[0]]
    L, T, F, S, A = ints(lengths), ints(table), ints(free), ints(state), ints([1] * R)
    o, p, r = (torch.empty(k, dtype=torch.int32, device=DEV) for k in ((R + 1,), (R,), (c.runs_for(R, R), 4)))
    c.extend(A, L.clone(), T.clone(), F.clone(), S.clone(), R)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.extend(A, L, T, F, S, R, offsets=o, positions=p, runs=r)
    want = (None, None, None, lengths, table, free, state)
    for _ in range(40):
        want = extend([1] * R, want[3], want[4], want[5], want[6], R, block, n, c.runs_for(R, R))
        graph.replay()
        torch.cuda.synchronize()
        assert [x.tolist() for x in (o, p, r, L, T, S)] == [want[0], want[1], want[2], want[3], want[4], want[6]]
