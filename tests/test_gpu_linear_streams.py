"""Calls with stream=: outputs that are allocated for them come from that stream's memory, and the results are those of the
current stream, whether the outputs are allocated or given."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen, offsets_of, quant_weight

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
def test_results_on_a_given_stream(raw):
    sizes, n, k = [40, 0, 200], 384, 512
    off, _ = offsets_of(sizes)
    rows = sum(sizes)
    x = torch.randn(rows, k, device=DEV, generator=gen(1)).bfloat16()
    dy = torch.randn(rows, n, device=DEV, generator=gen(2)).bfloat16()
    w = torch.randn(3 * n, k, device=DEV, generator=gen(3)) * 0.05
    bf, q8 = dr.Linear(w.bfloat16(), n_groups=3), dr.Linear(*quant_weight(w), n_groups=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on = side.cuda_stream if raw else side

    def run(stream, given=False):
        o = dict(stream=stream)
        e = [torch.zeros(r, c, dtype=t, device=DEV) for r, c, t in
             ((rows, k, torch.float8_e4m3fn), (4, rows, F32), (rows, n, BF16), (rows, n, BF16), (rows, k, BF16), (3 * n, k, F32))]
        torch.cuda.synchronize()
        q, s = dr.quant_rows(x, *(e[:2] if given else ()), **o)
        out = [dict(out=t) if given else {} for t in e[2:]]
        return [q.view(torch.uint8), s, q8.forward(q, s, off, **out[0], **o), bf.forward(x, None, off, **out[1], **o),
                bf.dgrad(dy, off, **out[2], **o), bf.wgrad(x, dy, off, **out[3], **o)]

    want = run(None)
    torch.cuda.synchronize()
    for given in (False, True):
        got = run(on, given)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_a_block_freed_on_the_current_stream_is_not_handed_to_another():
    x = torch.randn(64, 1 << 16, device=DEV, generator=gen(4)).bfloat16()  # 4 MB of codes: a block of its own
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    block = torch.empty(64, 1 << 16, dtype=torch.uint8, device=DEV)
    where = block.data_ptr()
    del block  # nothing is queued on it: the allocator may only give it to the current stream all the same
    codes, _ = dr.quant_rows(x, stream=side)
    side.synchronize()
    assert codes.data_ptr() != where
    again = torch.empty(64, 1 << 16, dtype=torch.uint8, device=DEV)
    assert again.data_ptr() == where
