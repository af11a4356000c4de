"""The test hook of the bounded waits refuses what would not restore itself."""
import paper_2607_22614_b200 as dr


def test_waits_hook_refuses():
    assert dr.dr_diag_linear_waits(2000001, 0) == dr.binding.DR_ERR_INVALID
    assert dr.dr_diag_linear_waits(0, 2) == dr.binding.DR_ERR_INVALID
    assert dr.dr_diag_linear_waits(0, 0) == 0
