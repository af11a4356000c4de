"""The tensor wrappers of the attention path on stand-in tensors: what they refuse and what they hand to the library, without a device and
without a launch; and the refusals of the C entry points that come before any device is asked."""
import ctypes as C

import pytest
import torch

import paper_2607_22614_b200 as dr
from test_linear_wrappers_host import E4M3, F32, I32, Stand, calls  # noqa: F401

B = dr.binding
BF16 = torch.bfloat16


@pytest.fixture
def made(calls, monkeypatch):  # noqa: F811
    monkeypatch.setattr(B, "dr_kv_cache_create", lambda desc: (calls.append(("dr_kv_cache_create", desc)), (0, C.c_void_p()))[1])
    monkeypatch.setattr(B, "dr_qk_create", lambda desc: (calls.append(("dr_qk_create", desc)), (0, C.c_void_p()))[1])
    monkeypatch.setattr(B, "dr_attend_work", lambda *a: (0, 4096))
    monkeypatch.setattr(B, "dr_qk_grad_work", lambda *a: (0, 4096))
    monkeypatch.setattr(B, "_empty", lambda r, c, dtype, device, stream: Flat(r, c, dtype=dtype))
    return calls


class Flat(Stand):
    def view(self, *_):
        return Flat(self.numel(), dtype=self.dtype, device=self.index)


class Bent(Stand):
    """Not contiguous."""

    def stride(self):
        return tuple(2 * s for s in super().stride())

    def is_contiguous(self):
        return False


class Stride4(Stand):
    def stride(self):
        return (1,) * len(self.shape)


def cache(**kw):
    return dr.KVCache(Stand(8, 2, 16, 64, dtype=E4M3, **kw), Stand(8, 2, 16, 64, dtype=E4M3, **kw), Stand(8, 2, dtype=F32, **kw), Stand(8, 2, dtype=F32, **kw))


def heads(**kw):
    return dr.QKHeads(4, 2, 64, Stand(64, **kw), Stand(64, **kw))


EXTEND = dict(added=(3, I32), lengths=(3, I32), table=(3, 5, I32), free=(8, I32), state=(2, I32), lengths_out=(3, I32), state_out=(2, I32), offsets=(4, I32),
              positions=(7, I32), runs=(6, 4, I32))
ATTEND = dict(q=(7, 256, BF16), lengths=(3, I32), table=(3, 5, I32), offsets=(4, I32), out=(7, 256, BF16))
FORWARD = dict(x=(7, 512, BF16), positions=(7, I32), out=(7, 384, BF16))
APPEND = dict(x=(7, 512, BF16), positions=(7, I32), runs=(6, 4, I32), out=(7, 256, BF16))
GRAD = dict(x=(7, 384, BF16), positions=(7, I32), dy=(7, 384, BF16), dx=(7, 384, BF16), dq_norm=(64, F32), dk_norm=(64, F32))


def stands(args, elsewhere=(), bent=()):
    out = {}
    for k, v in args.items():
        cls = Bent if k in bent else Stand
        out[k] = cls(*v[:-1], dtype=v[-1], device=int(k in elsewhere))
    return out


def call(which, args):
    if which is EXTEND:
        return cache().extend(rows=7, **args)
    if which is ATTEND:
        return cache().attend(**args)
    if which is FORWARD:
        return heads().forward(**args)
    if which is APPEND:
        return heads().append(cache=cache(), **args)
    return heads().grad(**args)


ALL = [EXTEND, ATTEND, FORWARD, APPEND, GRAD]
NAMES = ["dr_kv_extend", "dr_attend", "dr_qk_forward", "dr_qk_append", "dr_qk_grad"]


@pytest.mark.parametrize("which", range(5), ids=NAMES)
def test_the_stand_ins_pass(made, which):
    call(ALL[which], stands(ALL[which]))
    assert made[-1][0] == NAMES[which] and made[-1][1][-1] == 100  # the stream of GPU 0


@pytest.mark.parametrize("which,name", [(i, k) for i, a in enumerate(ALL) for k in a])
def test_operands_of_another_gpu_are_refused(made, which, name):
    with pytest.raises(ValueError, match="GPU 1"):
        call(ALL[which], stands(ALL[which], elsewhere=(name,)))
    assert made[-1][0] not in NAMES


@pytest.mark.parametrize("which,name", [(i, k) for i, a in enumerate(ALL) for k in a])
def test_operands_of_another_type_are_refused(made, which, name):
    args = stands(ALL[which])
    args[name] = Stand(*ALL[which][name][:-1], dtype=torch.float64)
    with pytest.raises((TypeError, ValueError)):
        call(ALL[which], args)
    assert made[-1][0] not in NAMES


@pytest.mark.parametrize("which,name", [(i, k) for i, a in enumerate(ALL) for k in a])
def test_operands_that_are_not_contiguous_are_refused(made, which, name):
    with pytest.raises(ValueError):
        call(ALL[which], stands(ALL[which], bent=(name,)))
    assert made[-1][0] not in NAMES


@pytest.mark.parametrize("which,name,shape", [
    (0, "added", (4,)), (0, "table", (2, 5)), (0, "free", (7,)), (0, "state", (1,)), (0, "offsets", (3,)), (0, "positions", (6,)), (0, "runs", (6, 3)),
    (0, "lengths_out", (4,)), (0, "state_out", (3,)), (1, "q", (7, 200)), (1, "q", (7, 64)), (1, "lengths", (4,)), (1, "table", (4, 5)), (1, "offsets", (3,)),
    (1, "out", (6, 256)), (2, "x", (7, 383)), (2, "positions", (6,)), (2, "out", (7, 512)), (3, "x", (7, 384)), (3, "out", (7, 384)),
    (4, "dy", (6, 384)), (4, "dy", (7, 512)), (4, "dx", (7, 256)), (4, "dq_norm", (63,))])
def test_operands_of_another_shape_are_refused(made, which, name, shape):
    args = stands(ALL[which])
    args[name] = Stand(*shape, dtype=ALL[which][name][-1])
    with pytest.raises(ValueError):
        call(ALL[which], args)
    assert made[-1][0] not in NAMES


@pytest.mark.parametrize("which,name", [(1, "q"), (2, "x"), (3, "x")])
def test_operands_that_autograd_would_follow_are_refused(made, which, name):
    args = stands(ALL[which])
    args[name] = Stand(*ALL[which][name][:-1], requires_grad=True)
    with pytest.raises(RuntimeError, match="gradient"):
        call(ALL[which], args)
    assert made[-1][0] not in NAMES
    with torch.no_grad():
        call(ALL[which], args)
    with pytest.raises(RuntimeError, match="gradient"):
        dr.QKHeads(4, 2, 64, Stand(64, requires_grad=True), Stand(64)).forward(**stands(FORWARD))


def test_other_arguments(made):
    with pytest.raises(ValueError, match="negative"):
        cache().attend(window=-1, **stands(ATTEND))
    with pytest.raises(ValueError, match="negative"):
        cache().attend(sinks=-1, **stands(ATTEND))
    with pytest.raises(ValueError, match="one row"):
        cache().attend(**{k: v for k, v in stands(ATTEND).items() if k != "offsets"})
    with pytest.raises(ValueError, match="accumulate"):
        heads().grad(accumulate=True, **{k: v for k, v in stands(GRAD).items() if k != "dq_norm"})
    with pytest.raises(ValueError, match="no gradients"):
        dr.QKHeads(4, 2, 64).grad(**stands(GRAD))
    with pytest.raises(ValueError, match="together"):
        dr.QKHeads(4, 2, 64, Stand(64))
    with pytest.raises(ValueError):
        cache().extend(rows=-1, **stands(EXTEND))


@pytest.mark.parametrize("k", [dict(dtype=torch.int8), dict(device=1), dict(shape=(8, 2, 16)), dict(shape=(8, 2, 16, 128))])
def test_caches_that_do_not_fit_together_are_refused(made, k):
    k = dict(dict(dtype=E4M3, device=0, shape=(8, 2, 16, 64)), **k)
    with pytest.raises(ValueError):
        dr.KVCache(Stand(8, 2, 16, 64, dtype=E4M3), Stand(*k["shape"], dtype=k["dtype"], device=k["device"]), Stand(8, 2, dtype=F32), Stand(8, 2, dtype=F32))
    with pytest.raises(ValueError):
        dr.KVCache(Stand(8, 2, 16, 64, dtype=E4M3), Stand(8, 2, 16, 64, dtype=E4M3), Stand(8, 3, dtype=F32), Stand(8, 2, dtype=F32))
    assert not made


# ---- the C entry points
def cache_desc(**kw):
    d = dict(struct_size=C.sizeof(B.dr_kv_cache_desc), n_blocks=4, kv_heads=2, block_tokens=16, head_dim=64, k_dev=4096, v_dev=8192, k_scale_dev=64,
             v_scale_dev=128)
    return B.dr_kv_cache_desc(**dict(d, **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=4), B.DR_ERR_INVALID), (dict(n_blocks=0), B.DR_ERR_INVALID), (dict(kv_heads=0), B.DR_ERR_INVALID), (dict(k_dev=None), B.DR_ERR_INVALID),
    (dict(v_scale_dev=None), B.DR_ERR_INVALID), (dict(block_tokens=48), B.DR_ERR_UNSUPPORTED), (dict(block_tokens=8), B.DR_ERR_UNSUPPORTED),
    (dict(head_dim=96), B.DR_ERR_UNSUPPORTED), (dict(n_blocks=1 << 27), B.DR_ERR_UNSUPPORTED), (dict(n_blocks=2 ** 32 - 1, kv_heads=2 ** 32 - 1), B.DR_ERR_UNSUPPORTED),
    (dict(k_dev=4104), B.DR_ERR_ALIGN), (dict(k_scale_dev=66), B.DR_ERR_ALIGN)])
def test_cache_descriptors_that_are_refused(kw, status):
    rc, h = B.dr_kv_cache_create(cache_desc(**kw))
    assert rc == status and not h and dr.dr_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=4), B.DR_ERR_INVALID), (dict(n_q_heads=0), B.DR_ERR_INVALID), (dict(n_kv_heads=0), B.DR_ERR_INVALID), (dict(k_norm_dev=None), B.DR_ERR_INVALID),
    (dict(eps=-1.0), B.DR_ERR_INVALID), (dict(eps=float("nan")), B.DR_ERR_INVALID), (dict(base=0.5), B.DR_ERR_INVALID), (dict(base=float("inf")), B.DR_ERR_INVALID),
    (dict(head_dim=32), B.DR_ERR_UNSUPPORTED), (dict(norm_dtype=B.DR_FP8_E4M3_B128), B.DR_ERR_UNSUPPORTED), (dict(n_q_heads=70000), B.DR_ERR_UNSUPPORTED),
    (dict(q_norm_dev=4097), B.DR_ERR_ALIGN)])
def test_head_descriptors_that_are_refused(kw, status):
    d = dict(struct_size=C.sizeof(B.dr_qk_desc), n_q_heads=4, n_kv_heads=2, head_dim=64, norm_dtype=B.DR_BF16, eps=1e-6, base=1e6, q_norm_dev=4096, k_norm_dev=8192)
    rc, h = B.dr_qk_create(B.dr_qk_desc(**dict(d, **kw)))
    assert rc == status and not h and dr.dr_last_error()


def test_null_handles():
    L = dr.lib()
    assert L.dr_kv_cache_create(None, None) == B.DR_ERR_INVALID and L.dr_qk_create(None, None) == B.DR_ERR_INVALID
    assert L.dr_kv_cache_destroy(None) == 0 and L.dr_qk_destroy(None) == 0
    assert B.dr_attend_work(None, 8, 1, 1)[0] == B.DR_ERR_INVALID and B.dr_qk_grad_work(None)[0] == B.DR_ERR_INVALID
    assert B.dr_kv_extend(None, *[None] * 3, 0, None, 0, 0, None, None, None, 0, None, None, None, 0, None) == B.DR_ERR_INVALID
    assert B.dr_qk_forward(None, None, B.DR_BF16, 0, None, 0, None, 0, None) == B.DR_ERR_INVALID
    assert B.dr_attend(None, None, 0, 8, 0, None, None, 0, None, 0, 0, 1.0, 0, 0, None, 0, None, 0, None) == B.DR_ERR_INVALID


def test_calls_by_words():
    """dr_call has the entry points' own checks, and every packed form has as many words as its entry point has arguments."""
    import struct
    assert B.dr_call(0, None) == B.DR_ERR_INVALID and B.dr_call(5, bytes(200)) == B.DR_ERR_INVALID
    for name, (what, form) in B._PACKED.items():
        args = getattr(dr.lib(), name).argtypes
        assert struct.calcsize(form) == 8 * len(args), name
        assert B.dr_call(what, bytes(8 * len(args))) == B.DR_ERR_INVALID  # no handle
        assert B._fn(name)(*[0] * len(args)) == B.DR_ERR_INVALID
