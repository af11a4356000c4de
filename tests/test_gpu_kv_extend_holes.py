"""Requests that end with blocks that they do not hold any more: entries outside the cache, say behind a window."""
import random

import pytest
import torch

import paper_2607_22614_b200 as dr
from attend_util import extend
from test_gpu_kv_extend import cache, ints

pytestmark = pytest.mark.gpu


def returned(added, lengths, table, free, state, block, n_blocks):
    """What comes back, block by block: the free list and how many it holds before any is taken."""
    free, count = list(free), state[0]
    for r, a in enumerate(added):
        for b in table[r][:-(-lengths[r] // block)] if a < 0 else []:
            if 0 <= b < n_blocks:
                free[count] = b
                count += 1
    return free, count


@pytest.mark.parametrize("requests,width,block", [(1, 5, 16), (3, 700, 16), (64, 40, 128), (600, 24, 16), (1500, 3, 32)])
@pytest.mark.parametrize("given", [0.0, 0.3, 0.97])
@pytest.mark.parametrize("prompts", [False, True])
def test_only_blocks_that_are_held_come_back(requests, width, block, given, prompts):
    """The new requests' blocks come out of those: none of them lies outside the cache, and none is lost."""
    rng = random.Random(requests + int(100 * given))
    ids = list(range(requests * width + 9))
    rng.shuffle(ids)
    n, lengths, table = len(ids), [], []
    for _ in range(requests):
        lengths.append(rng.randint(0, width * block))
        need = -(-lengths[-1] // block)
        row = [ids.pop() for _ in range(need)] + [-1] * (width - need)
        for j in range(need):
            if rng.random() < given:
                ids.append(row[j])
                row[j] = rng.choice([-1, n, -2 ** 31, 2 ** 31 - 1])
        table.append(row)
    free, state = ids + [-9] * (n - len(ids)), [len(ids), 0]
    added = [rng.choice([-1, -1, 0, 2 * block if prompts else 1]) for _ in range(requests)]
    rows = sum(max(a, 0) for a in added)
    c = cache(n, block)
    L, T, F, S = ints(lengths), ints(table), ints(free), ints(state)
    o, p, r = c.extend(ints(added), L, T, F, S, rows)
    free, count = returned(added, lengths, table, free, state, block, n)
    # the rest of the step is that of the same requests without the ends, over the list as it is then
    held = [0 if a < 0 else m for a, m in zip(added, lengths)]
    w = extend([max(a, 0) for a in added], held, table, free, [count, 0], rows, block, n, c.runs_for(requests, rows))
    assert [x.tolist() for x in (o, p, r, L, T, S)] == [w[0], w[1], w[2], w[3], w[4], w[6]]
    left = F[:int(S[0])].tolist()
    assert left == free[:int(S[0])]
    owned = [b for i, a in enumerate(added) if a >= 0 for b in T[i, :-(-int(L[i]) // block)].tolist() if 0 <= b < n]
    assert sorted(owned + left) == list(range(n))
