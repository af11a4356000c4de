"""Row pitches that the products refuse, next to the ones that they take (no launch happens for a refused call)."""
import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV, check, gen, product

pytestmark = pytest.mark.gpu
B, BF16 = dr.binding, dr.DR_BF16


def test_products_refuse_pitches_out_of_range():
    layer = dr.Linear(torch.zeros(128, 128, dtype=torch.bfloat16, device=DEV))
    x, y = (torch.zeros(4, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dw = torch.zeros(128, 128, device=DEV)
    h, p, q, w = layer.handle, x.data_ptr(), y.data_ptr(), dw.data_ptr()
    for big in ((1 << 40) + 8, 1 << 62, 1 << 63, (1 << 64) - 8):
        assert B.dr_linear_forward(h, p, big, None, 0, 4, None, q, 128, BF16, None) == B.DR_ERR_INVALID
        assert B.dr_linear_forward(h, p, 128, None, 0, 4, None, q, big, BF16, None) == B.DR_ERR_INVALID
        assert B.dr_linear_dgrad(h, p, big, 4, None, q, 128, BF16, None) == B.DR_ERR_INVALID
        assert B.dr_linear_dgrad(h, p, 128, 4, None, q, big, BF16, None) == B.DR_ERR_INVALID
        assert B.dr_linear_wgrad(h, p, big, q, 128, 4, None, w, 128, 0, None) == B.DR_ERR_INVALID
        assert B.dr_linear_wgrad(h, p, 128, q, big, 4, None, w, 128, 0, None) == B.DR_ERR_INVALID
        assert B.dr_linear_wgrad(h, p, 128, q, 128, 4, None, w, big, 0, None) == B.DR_ERR_INVALID
    # 2^30 rows of 2^31 elements: each pitch is in range, the rows together are not
    assert B.dr_linear_forward(h, p, 1 << 31, None, 0, 1 << 30, None, q, 128, BF16, None) == B.DR_ERR_INVALID
    q8 = dr.Linear(torch.zeros(128, 256, dtype=torch.float8_e4m3fn, device=DEV), torch.ones(1, 2, device=DEV))
    assert B.dr_linear_forward(q8.handle, p, 256, p, 1 << 62, 4, None, q, 128, BF16, None) == B.DR_ERR_INVALID


def test_one_row_may_have_any_pitch_in_range():
    x = torch.randn(1, 128, device=DEV, generator=gen(1)).bfloat16()
    w = torch.randn(64, 128, device=DEV, generator=gen(2)).bfloat16()
    layer, y = dr.Linear(w), torch.empty(1, 64, dtype=torch.bfloat16, device=DEV)
    for ldx, ldy in ((128, 64), (1 << 20, 1 << 40), (1 << 40, 1 << 20)):
        y.zero_()
        rc = B.dr_linear_forward(layer.handle, x.data_ptr(), ldx, None, 0, 1, None, y.data_ptr(), ldy, BF16,
                                 torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        want, tol = product(x.double(), w.double().t(), torch.bfloat16)
        check(y, want, tol)
