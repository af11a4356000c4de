"""Windows and first tokens beyond 2^30, over lengths beyond it."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen

pytestmark = pytest.mark.gpu
BLOCK, DIM, FAR = 128, 64, 1 << 30


def far_cache():
    """One head; blocks 0 .. 3 of normal values, and a table of 2^23 + 2^13 blocks that holds none but what the tests put there."""
    k, v = (torch.randn(4, 1, BLOCK, DIM, device=DEV, generator=gen(i)).to(torch.float8_e4m3fn) for i in (1, 2))
    ones = torch.ones(4, 1, device=DEV)
    table = torch.full((1, (1 << 23) + (1 << 13)), -1, dtype=torch.int32, device=DEV)
    return k, v, dr.KVCache(k, v, ones, ones.clone()), table


def plain(q, k, v, tokens):
    """Attention to the four blocks' tokens of those numbers in 64 bits, and its error: logits of a few units are off by 2^-17 at most, a p
    by 2^-11 (fp16) and the exponential's 2^-18, doubled for their sum, the result by 2^-8."""
    kk, vv = k.double().view(-1, DIM)[tokens], v.double().view(-1, DIM)[tokens]
    p = torch.softmax(DIM ** -0.5 * q.double() @ kk.t(), 1)
    return p @ vv, 2.0 ** -8 * (p @ vv).abs() + 2 * (2.0 ** -11 + 2.0 ** -16) * (p @ vv.abs())


@pytest.mark.parametrize("window,sinks,first", [(FAR + 5, 0, None), (FAR + 5, 70, 70), (2 ** 31 - 2, 3, 128), (2 ** 31 - 1, 0, 128), (1 << 63, 0, 128),
                                                (1 << 40, 1 << 40, 128), (300, FAR + 200, 128), (300, 3, 3)])
def test_far_windows(window, sinks, first):
    """`first`: how many of the first block's tokens are seen (the last two blocks', which end the request, are)."""
    k, v, cache, table = far_cache()
    n = FAR + (1 << 20)
    table[0, 0], table[0, n // BLOCK - 2], table[0, n // BLOCK - 1] = 0, 1, 2
    if sinks > FAR:  # a block that only sinks reach
        table[0, FAR // BLOCK] = 3
    q = torch.randn(1, DIM, device=DEV, generator=gen(3)).bfloat16()
    got = cache.attend(q, torch.tensor([n], dtype=torch.int32, device=DEV), table, window=window, sinks=sinks)
    tokens = list(range(first or 0)) + list(range(128, 384)) + (list(range(384, 512)) if sinks > FAR else [])
    want, tol = plain(q, k, v, tokens)
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("added", [5, 160])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 2, 0), (2 ** 31 - 2, 2 ** 31 - 1), (1 << 40, 1 << 40)])
def test_rows_before_the_first_token_under_a_far_window(added, window, sinks):
    _, _, cache, table = far_cache()
    table = table[:, :2].clone()
    table[0, 0] = 1
    q = torch.randn(added, DIM, device=DEV, generator=gen(4)).bfloat16()
    L, offsets = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([3], [0, added]))
    want = cache.attend(q, L, table, offsets)
    assert (want[:added - 3] == 0).all() and (want[added - 3:] != 0).any(1).all()
    assert torch.equal(cache.attend(q, L, table, offsets, window=window, sinks=sinks), want)
