"""Row pitches of the linear-layer entry points at the edge of 64-bit offsets: sizes that only fit because a product of rows
and pitch wrapped around are refused.  No device is needed; no refused call reads its pointers."""
import ctypes as C

import pytest

import paper_2607_22614_b200 as dr

B = dr.binding
P = 1 << 20
BF16, FP8 = dr.DR_BF16, dr.DR_FP8_E4M3_B128


def _create(**kw):
    d = dict(struct_size=C.sizeof(dr.dr_linear_desc), dtype=BF16, n_groups=1, out_features=8, in_features=16, weight_dev=P)
    d.update(kw)
    return dr.dr_linear_create(dr.dr_linear_desc(**d))[0]


@pytest.mark.parametrize("kw,status", [
    # 2^24 rows after the first, 2^40 elements apart, two bytes each: 2^65 bytes, which is 0 in 64 bits
    (dict(out_features=(1 << 24) + 1, weight_ld=1 << 40, weight_bytes=32), B.DR_ERR_INVALID),
    (dict(out_features=(1 << 24) + 1, weight_ld=1 << 40, weight_bytes=(1 << 64) - 1), B.DR_ERR_INVALID),
    (dict(out_features=1 << 30, weight_ld=1 << 34, weight_bytes=32), B.DR_ERR_INVALID),
    (dict(out_features=(1 << 20) + 1, weight_ld=1 << 40, weight_bytes=(1 << 61) + 31), B.DR_ERR_SIZE),
    (dict(out_features=(1 << 20) + 1, weight_ld=1 << 40, weight_bytes=32), B.DR_ERR_SIZE),
    # scales: 2^24 rows of blocks need 2^31 rows; 2^22 rows of scales after the first, 2^40 floats apart: 2^64 bytes
    (dict(dtype=FP8, out_features=(1 << 29) + 1, weight_bytes=1 << 40, scale_dev=P, scale_ld=1 << 40, scale_bytes=4), B.DR_ERR_INVALID),
    (dict(dtype=FP8, out_features=(1 << 27) + 1, weight_bytes=1 << 40, scale_dev=P, scale_ld=1 << 40, scale_bytes=4), B.DR_ERR_SIZE),
    (dict(weight_ld=(1 << 40) + 16, weight_bytes=(1 << 64) - 1), B.DR_ERR_INVALID)])
def test_create_refuses_what_wraps(kw, status):
    assert _create(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(ldx=(1 << 40) + 1), B.DR_ERR_INVALID), (dict(ldx=1 << 63), B.DR_ERR_INVALID), (dict(ldc=1 << 63), B.DR_ERR_INVALID),
    (dict(lds=1 << 62, cols=129, ldx=129, ldc=129), B.DR_ERR_INVALID), (dict(rows=1 << 30, src=1 << 30, lds=1 << 30, ldx=1 << 31), B.DR_ERR_INVALID),
    (dict(rows=1 << 30, src=1 << 30, lds=1 << 30, ldc=1 << 31), B.DR_ERR_INVALID), (dict(rows=0, ldx=1 << 40), 0)])
def test_quant_rows_refuses_what_wraps(kw, status):
    a = dict(x=P, x_dtype=BF16, ldx=64, src=4, index=None, form=0, rows=4, cols=64, codes=P, ldc=64, scales=P, lds=4)
    a.update(kw)
    assert dr.dr_quant_rows(*a.values(), None) == status



@pytest.mark.parametrize("kw,status", [
    (dict(out_features=(1 << 31) - 511), B.DR_ERR_UNSUPPORTED), (dict(in_features=(1 << 31) - 511), B.DR_ERR_UNSUPPORTED),
    (dict(n_groups=(1 << 31) - 511, out_features=1), B.DR_ERR_UNSUPPORTED), (dict(n_groups=2, out_features=(1 << 30) - 255), B.DR_ERR_UNSUPPORTED),
    (dict(out_features=(1 << 31) - 512), B.DR_ERR_SIZE), (dict(in_features=(1 << 31) - 512), B.DR_ERR_SIZE),
    (dict(n_groups=2, out_features=(1 << 30) - 256), B.DR_ERR_SIZE)])
def test_features_leave_room_for_the_last_tiles(kw, status):
    """The kernels' tiles end up to two tiles past the last feature, which they count in int."""
    assert _create(**kw, weight_bytes=64) == status
