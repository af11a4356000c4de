"""Products and quantisations that follow each other on one stream without a wait of the host: every kernel starts while the one
before it still writes, and must read nothing of it too early."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, gen, quant_weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 7, 300])
@pytest.mark.parametrize("cols", [1024, 272, 264, 257])  # whole groups of sixteen, of eight, and none
def test_chain_over_reused_buffers(cols, rows, fp32):
    hidden, g = 512, gen(cols + rows)
    up = dr.Linear(*quant_weight(torch.randn(2 * cols, hidden, device=DEV, generator=g) * 0.05))
    down = dr.Linear(*quant_weight(torch.randn(hidden, cols, device=DEV, generator=g) * 0.05))
    inputs = [torch.randn(rows, hidden, device=DEV, generator=g).bfloat16() for _ in range(8)]
    x = torch.empty_like(inputs[0])
    h = torch.empty(rows, 2 * cols, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
    y = torch.empty(rows, hidden, dtype=torch.bfloat16, device=DEV)
    xq, xs = dr.quant_rows(inputs[0])
    hq, hs = dr.quant_rows(h.zero_(), swiglu=True)

    def chain(between=None):
        out = []
        if between is None:  # the host gets ahead meanwhile, so that the kernels follow each other without a gap
            torch.cuda._sleep(20_000_000)
        for v in inputs * 4:
            x.copy_(v)
            for step in (lambda: dr.quant_rows(x, xq, xs), lambda: up.forward(xq, xs, out=h),
                         lambda: dr.quant_rows(h, hq, hs, swiglu=True), lambda: down.forward(hq, hs, out=y),
                         lambda: dr.quant_rows(y, xq, xs), lambda: up.forward(xq, xs, out=h)):
                step()
                if between:
                    between()
            out.append((h.clone(), y.clone(), hq.clone(), hs.clone()))
        torch.cuda.synchronize()
        return out

    want, got = chain(torch.cuda.synchronize), chain()
    for a, b in zip(want, got):
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a, b))
