"""Refusals of the linear-layer entry points that need no device."""
import ctypes as C

import pytest

import paper_2607_22614_b200 as dr

B = dr.binding
P = 1 << 20  # a non-NULL address that no refused call reads


def _desc(**kw):
    d = dict(struct_size=C.sizeof(dr.dr_linear_desc), dtype=dr.DR_BF16, n_groups=2, out_features=8, in_features=16, weight_dev=P,
             weight_bytes=2 * 8 * 16 * 2)
    d.update(kw)
    return dr.dr_linear_desc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), B.DR_ERR_INVALID), (dict(dtype=dr.DR_F32), B.DR_ERR_UNSUPPORTED), (dict(dtype=9), B.DR_ERR_UNSUPPORTED),
    (dict(n_groups=0), B.DR_ERR_INVALID), (dict(out_features=0), B.DR_ERR_INVALID), (dict(in_features=0), B.DR_ERR_INVALID),
    (dict(out_features=1 << 31), B.DR_ERR_UNSUPPORTED), (dict(out_features=1 << 30), B.DR_ERR_UNSUPPORTED),
    (dict(in_features=1 << 31), B.DR_ERR_UNSUPPORTED), (dict(weight_dev=None), B.DR_ERR_INVALID), (dict(scale_dev=P), B.DR_ERR_INVALID),
    (dict(dtype=dr.DR_FP8_E4M3_B128), B.DR_ERR_INVALID), (dict(weight_ld=15), B.DR_ERR_INVALID), (dict(weight_ld=1 << 50), B.DR_ERR_INVALID),
    (dict(weight_dev=P + 1), B.DR_ERR_ALIGN), (dict(weight_bytes=511), B.DR_ERR_SIZE), (dict(weight_ld=17), B.DR_ERR_SIZE),
    (dict(dtype=dr.DR_FP8_E4M3_B128, scale_dev=P, scale_bytes=3), B.DR_ERR_SIZE),
    (dict(dtype=dr.DR_FP8_E4M3_B128, scale_dev=P + 2, scale_bytes=64), B.DR_ERR_ALIGN),
    (dict(dtype=dr.DR_FP8_E4M3_B128, scale_dev=P, scale_bytes=64, in_features=300, weight_bytes=1 << 20, scale_ld=2), B.DR_ERR_INVALID)])
def test_create_refuses(kw, status):
    rc, h = dr.dr_linear_create(_desc(**kw))
    assert rc == status and not h.value and dr.dr_last_error()


def test_null_handles():
    assert dr.dr_linear_destroy(None) == 0
    assert dr.dr_linear_forward(None, P, 16, None, 0, 1, None, P, 8, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert dr.dr_linear_dgrad(None, P, 8, 1, None, P, 16, dr.DR_BF16, None) == B.DR_ERR_INVALID
    assert dr.dr_linear_wgrad(None, P, 16, P, 8, 1, None, P, 16, 0, None) == B.DR_ERR_INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(x_dtype=7), B.DR_ERR_UNSUPPORTED), (dict(form=2), B.DR_ERR_UNSUPPORTED), (dict(rows=1 << 31, src=1 << 31, lds=1 << 31), B.DR_ERR_UNSUPPORTED),
    (dict(cols=0), B.DR_ERR_INVALID), (dict(ldx=63), B.DR_ERR_INVALID), (dict(ldc=63), B.DR_ERR_INVALID), (dict(lds=3), B.DR_ERR_INVALID),
    (dict(src=3), B.DR_ERR_INVALID), (dict(form=1), B.DR_ERR_INVALID), (dict(x=None), B.DR_ERR_INVALID), (dict(codes=None), B.DR_ERR_INVALID),
    (dict(scales=None), B.DR_ERR_INVALID), (dict(x=P + 1), B.DR_ERR_ALIGN), (dict(scales=P + 2), B.DR_ERR_ALIGN),
    (dict(index=P + 4), B.DR_ERR_ALIGN), (dict(rows=0), 0)])
def test_quant_rows_refuses(kw, status):
    a = dict(x=P, x_dtype=dr.DR_BF16, ldx=64, src=4, index=None, form=0, rows=4, cols=64, codes=P, ldc=64, scales=P, lds=4)
    a.update(kw)
    assert dr.dr_quant_rows(*a.values(), None) == status
