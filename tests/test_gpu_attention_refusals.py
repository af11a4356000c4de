"""What the attention path's C entry points refuse before they launch, with live handles."""
import ctypes as C

import pytest
import torch

import paper_2607_22614_b200 as dr
from linear_util import DEV

pytestmark = pytest.mark.gpu
B = dr.binding
K = 1 << 20


@pytest.fixture(scope="module")
def live():
    """A cache, heads with norms and without, and memory to point at (nothing of it is used: every call is refused)."""
    cache, w = dr.KVCache.empty(8, 2, 16, 64), torch.ones(64, device=DEV)
    memory = torch.zeros(K, dtype=torch.uint8, device=DEV)
    return cache, dr.QKHeads(4, 2, 64, w, w), dr.QKHeads(4, 3, 64), memory


def refused(fn, good, changes):
    for kw, status in changes:
        args = dict(good, **kw)
        rc = fn(*args.values())
        assert rc == status and dr.dr_last_error(), (kw, rc, dr.dr_last_error())


def test_extend(live):
    cache, _, _, m = live
    p = m.data_ptr()
    good = dict(cache=cache.handle, added=p, lengths=p, lengths_out=p, requests=3, table=p, ld_table=5, width=5, free_list=p, state=p, state_out=p, rows=7,
                offsets=p, positions=p, runs=p, n_runs=6, stream=None)
    nulls = [({k: None}, B.DR_ERR_INVALID) for k in ("added", "lengths", "lengths_out", "table", "free_list", "state", "state_out", "offsets", "positions", "runs")]
    odd = [({k: p + 2}, B.DR_ERR_ALIGN) for k in ("added", "lengths", "lengths_out", "table", "free_list", "state", "state_out", "offsets", "positions")]
    refused(dr.dr_kv_extend, good, nulls + odd + [
        (dict(runs=p + 4), B.DR_ERR_ALIGN), (dict(ld_table=4), B.DR_ERR_INVALID), (dict(width=0), B.DR_ERR_INVALID), (dict(n_runs=5), B.DR_ERR_SIZE),
        (dict(requests=1 << 25), B.DR_ERR_UNSUPPORTED), (dict(rows=1 << 31), B.DR_ERR_UNSUPPORTED), (dict(width=1 << 25, ld_table=1 << 25), B.DR_ERR_UNSUPPORTED)])


def test_heads(live):
    cache, heads, other, m = live
    p = m.data_ptr()
    good = dict(qk=heads.handle, x=p, dtype=B.DR_BF16, ldx=384, positions=p, rows=7, y=p, ldy=384, stream=None)
    changes = [({k: None}, B.DR_ERR_INVALID) for k in ("x", "positions", "y")] + [
        (dict(dtype=B.DR_FP8_E4M3_B128), B.DR_ERR_UNSUPPORTED), (dict(ldx=383), B.DR_ERR_INVALID), (dict(ldy=383), B.DR_ERR_INVALID),
        (dict(ldx=1 << 41), B.DR_ERR_INVALID), (dict(rows=1 << 31), B.DR_ERR_UNSUPPORTED), (dict(x=p + 1), B.DR_ERR_ALIGN), (dict(positions=p + 2), B.DR_ERR_ALIGN)]
    refused(dr.dr_qk_forward, good, changes)
    good = dict(qk=heads.handle, x=p, dtype=B.DR_BF16, ldx=512, positions=p, rows=7, runs=p, n_runs=3, cache=cache.handle, y=p, ldy=256, stream=None)
    refused(dr.dr_qk_append, good, [({k: None}, B.DR_ERR_INVALID) for k in ("x", "positions", "y", "runs", "cache")] + [
        (dict(ldx=511), B.DR_ERR_INVALID), (dict(ldy=255), B.DR_ERR_INVALID), (dict(runs=p + 4), B.DR_ERR_ALIGN), (dict(n_runs=1 << 31), B.DR_ERR_UNSUPPORTED),
        (dict(qk=other.handle, ldx=640), B.DR_ERR_INVALID)])
    rc, need = dr.dr_qk_grad_work(heads.handle)
    assert rc == 0 and 0 < need <= K and dr.dr_qk_grad_work(other.handle) == (0, 0)
    good = dict(qk=heads.handle, x=p, dtype=B.DR_F32, ldx=384, positions=p, dy=p, lddy=384, rows=7, dx=p, lddx=384, dq=p, dk=p, accumulate=0, work=p,
                work_bytes=need, stream=None)
    refused(dr.dr_qk_grad, good, [({k: None}, B.DR_ERR_INVALID) for k in ("x", "positions", "dy", "dx", "dq", "dk")] + [
        (dict(work=None), B.DR_ERR_SIZE), (dict(work_bytes=need - 1), B.DR_ERR_SIZE), (dict(work=p + 8), B.DR_ERR_ALIGN), (dict(accumulate=2), B.DR_ERR_INVALID),
        (dict(lddy=383), B.DR_ERR_INVALID), (dict(lddx=383), B.DR_ERR_INVALID), (dict(dq=p + 2), B.DR_ERR_ALIGN), (dict(dy=p + 2), B.DR_ERR_ALIGN)])


def test_attend(live):
    cache, _, _, m = live
    p = m.data_ptr()
    rc, need = dr.dr_attend_work(cache.handle, 8, 3, 7)
    assert rc == 0 and need > 0
    work = torch.zeros(need, dtype=torch.uint8, device=DEV)
    good = dict(cache=cache.handle, q=p, ldq=512, n_q_heads=8, rows=7, offsets=p, lengths=p, requests=3, table=p, ld_table=500, width=500, scale=0.1, window=0,
                sinks=0, out=p, ldo=512, work=work.data_ptr(), work_bytes=need, stream=None)
    refused(dr.dr_attend, good, [({k: None}, B.DR_ERR_INVALID) for k in ("q", "lengths", "table", "out")] + [
        (dict(n_q_heads=7), B.DR_ERR_INVALID), (dict(n_q_heads=0), B.DR_ERR_INVALID), (dict(n_q_heads=130, ldq=9000, ldo=9000), B.DR_ERR_UNSUPPORTED),
        (dict(offsets=None), B.DR_ERR_INVALID), (dict(scale=float("nan")), B.DR_ERR_INVALID), (dict(scale=float("inf")), B.DR_ERR_INVALID),
        (dict(ldq=511), B.DR_ERR_INVALID), (dict(ldo=511), B.DR_ERR_INVALID), (dict(ld_table=499), B.DR_ERR_INVALID), (dict(width=0), B.DR_ERR_INVALID),
        (dict(work=None), B.DR_ERR_SIZE), (dict(work_bytes=need - 1), B.DR_ERR_SIZE), (dict(work=work.data_ptr() + 8), B.DR_ERR_ALIGN), (dict(q=p + 1), B.DR_ERR_ALIGN),
        (dict(lengths=p + 2), B.DR_ERR_ALIGN), (dict(requests=1 << 25), B.DR_ERR_UNSUPPORTED), (dict(rows=1 << 31), B.DR_ERR_UNSUPPORTED),
        (dict(width=1 << 25, ld_table=1 << 25), B.DR_ERR_UNSUPPORTED)])


def test_nothing_to_do(live):
    cache, heads, _, m = live
    p, w = m.data_ptr(), torch.zeros(dr.dr_attend_work(cache.handle, 8, 0, 0)[1], dtype=torch.uint8, device=DEV)
    assert dr.dr_attend(cache.handle, p, 512, 8, 0, p, p, 3, p, 5, 5, 0.1, 0, 0, p, 512, w.data_ptr(), w.numel(), None) == 0
    assert dr.dr_qk_append(heads.handle, p, B.DR_BF16, 512, p, 0, p, 0, cache.handle, p, 256, None) == 0
    torch.cuda.synchronize()
