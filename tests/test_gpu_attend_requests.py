"""Steps of many requests that mix prompts, drafts, single tokens and idle ones, with offsets."""
import pytest
import torch

from test_gpu_attend import check, setup

pytestmark = pytest.mark.gpu


def step(requests, prompts, idle):
    """New tokens of each request: prompts at some, none at others, one or five at the rest."""
    return [(70 + 23 * (i % 11) if i in prompts else 0 if i in idle else (1, 5, 1)[i % 3]) for i in range(requests)]


@pytest.mark.parametrize("requests,prompts,idle", [
    (127, {0, 64, 126}, set()), (128, {127}, {5}), (129, {128}, set(range(0, 128, 2))), (129, {0, 3, 128}, set()),
    (513, {512}, set(range(160, 480))),          # the only prompt in the second chunk of 512; chunks of 160 without rows
    (513, {3, 511}, set(range(512))),
    (1100, {1, 500, 1024, 1060, 1099}, set(range(320, 640)) | {1098}),  # a chunk of 512 without prompts
    (1100, set(range(600, 640)), set(range(0, 600))),
    (1100, set(), set(range(1, 1100))),
    (700, set(range(700)), set()),
])
def test_mixed_steps(requests, prompts, idle):
    added = step(requests, prompts, idle)
    lengths = [a + (i * 37) % 90 for i, a in enumerate(added)]
    q, cache, table, offsets = setup(requests, lengths, added, 4, 2, 64, 32, garbage=False)
    check(q, cache, table, lengths, offsets, 4)


def test_mixed_steps_of_long_requests():
    """Unlike lengths, so that the order by length is not the order of the requests, and groups that several CTAs have."""
    added = [1, 300, 5, 0, 1, 90, 1, 8, 200, 1] * 16
    lengths = [a + (i * 977) % 4000 for i, a in enumerate(added)]
    q, cache, table, offsets = setup(5, lengths, added, 4, 1, 128, 128, garbage=False)
    check(q, cache, table, lengths, offsets, 4)
