"""The tensor wrappers of the linear layers on stand-in tensors: what they refuse and what they hand to the library, without a device
and without a launch."""
import ctypes as C

import pytest
import torch

import paper_2607_22614_b200 as dr

B = dr.binding
SIZES = {torch.bfloat16: 2, torch.float32: 4, torch.int32: 4, torch.int64: 8, torch.float64: 8}


class Stand:
    """What the wrappers look at in a contiguous CUDA tensor."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, requires_grad=False):
        self.shape, self.dtype, self.index, self.requires_grad = shape, dtype, device, requires_grad
        self.is_cuda, self.device = True, torch.device("cuda", device)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def is_contiguous(self):
        return True

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return SIZES.get(self.dtype, 1)

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def calls(monkeypatch):
    """GPU 0 is current; the library's calls are noted instead of made."""
    made = []

    def fn(name):
        def call(*args):
            made.append((name, args))
            return 0
        return call

    def create(desc):
        made.append(("dr_linear_create", desc))
        return 0, C.c_void_p()  # (NULL: nothing to destroy)

    monkeypatch.setattr(B, "_fn", fn)
    monkeypatch.setattr(B, "dr_linear_create", create)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(B, "_raw_stream", lambda index: 100 + index)
    return made


E4M3 = torch.float8_e4m3fn
F32, I32, I64 = torch.float32, torch.int32, torch.int64


def _layer(groups=2, fp8=False, **kw):
    if fp8:
        return dr.Linear(Stand(groups * 128, 256, dtype=E4M3, **kw), Stand(groups, 2, dtype=F32, **kw), n_groups=groups)
    return dr.Linear(Stand(groups * 128, 256, **kw), n_groups=groups)


def test_the_stand_ins_pass(calls):
    bf, q8, off = _layer(), _layer(fp8=True), Stand(3, dtype=I32)
    bf.forward(Stand(5, 256), None, off, out=Stand(5, 128))
    q8.forward(Stand(5, 256, dtype=E4M3), Stand(2, 5, dtype=F32), off, out=Stand(5, 128))
    bf.dgrad(Stand(5, 128), off, out=Stand(5, 256))
    bf.wgrad(Stand(5, 256), Stand(5, 128), off, out=Stand(256, 256, dtype=F32))
    dr.quant_rows(Stand(5, 256), Stand(4, 256, dtype=E4M3), Stand(2, 4, dtype=F32), row_index=Stand(4, dtype=I64))
    assert [c[0] for c in calls] == ["dr_linear_create"] * 2 + ["dr_linear_forward"] * 2 + ["dr_linear_dgrad", "dr_linear_wgrad",
                                                                                           "dr_quant_rows"]
    assert all(c[1][-1] == 100 for c in calls[2:])  # the stream of GPU 0


QUANT = dict(x=(5, 256), codes=(4, 256, E4M3), scales=(2, 4, F32), row_index=(4, I64))
FORWARD = dict(x=(5, 256, E4M3), x_scale=(2, 5, F32), offsets=(3, I32), out=(5, 128, torch.bfloat16))
DGRAD = dict(dy=(5, 128), offsets=(3, I32), out=(5, 256))
WGRAD = dict(x=(5, 256), dy=(5, 128), offsets=(3, I32), out=(256, 256, F32))


def _stands(args, elsewhere):
    out = {}
    for k, v in args.items():
        dtype = v[-1] if isinstance(v[-1], torch.dtype) else torch.bfloat16
        out[k] = Stand(*[s for s in v if isinstance(s, int)], dtype=dtype, device=int(k in elsewhere))
    return out


@pytest.mark.parametrize("args,which", [(a, w) for a in (QUANT, FORWARD, DGRAD, WGRAD) for w in list(a) + ["all"]])
def test_operands_of_another_gpu_are_refused(calls, args, which):
    layer = _layer(fp8=args is FORWARD)
    call = dr.quant_rows if args is QUANT else getattr(layer, {id(FORWARD): "forward", id(DGRAD): "dgrad", id(WGRAD): "wgrad"}[id(args)])
    del calls[:]
    with pytest.raises(ValueError, match="GPU 1"):
        call(**_stands(args, list(args) if which == "all" else [which]))
    assert not calls


def test_a_layer_of_another_gpu_is_refused(calls):
    for kw in (dict(weight=Stand(128, 256, device=1)), dict(weight=Stand(128, 256, dtype=E4M3, device=1), scale=Stand(1, 2, dtype=F32, device=1)),
               dict(weight=Stand(128, 256, dtype=E4M3), scale=Stand(1, 2, dtype=F32, device=1))):
        with pytest.raises(ValueError, match="GPU 1"):
            dr.Linear(**kw)
    assert not calls


@pytest.mark.parametrize("given", [False, True], ids=["allocated", "given"])
@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
def test_allocated_outputs_belong_to_the_stream_of_the_call(calls, monkeypatch, raw, given):
    """Memory that the current stream has freed may still be in use there: another stream must not be handed it."""
    entered, made_in = [], []

    class Stream:
        def __init__(self, handle, device=None):
            self.cuda_stream = handle

    class Under:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream.cuda_stream)

        def __exit__(self, *_):
            entered.pop()

    def empty(*shape, dtype, device):
        made_in.append(entered[-1] if entered else "current")
        return Stand(*shape, dtype=dtype)

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", Under)
    layer, off = _layer(), Stand(3, dtype=I32)
    del calls[:]
    for at in (None, 77 if raw else Stream(77)):
        kw = [dict(stream=at) for _ in range(4)]
        if given:
            kw[0].update(codes=Stand(5, 256, dtype=E4M3), scales=Stand(2, 5, dtype=F32))
            kw[1].update(out=Stand(5, 128))
            kw[2].update(out=Stand(5, 256))
            kw[3].update(out=Stand(256, 256, dtype=F32))
        dr.quant_rows(Stand(5, 256), **kw[0])
        layer.forward(Stand(5, 256), None, off, **kw[1])
        layer.dgrad(Stand(5, 128), off, **kw[2])
        layer.wgrad(Stand(5, 256), Stand(5, 128), off, **kw[3])
    assert made_in == ([] if given else ["current"] * 5 + [77] * 5)
    assert [c[1][-1] for c in calls] == [100] * 4 + [77] * 4


BYTES = [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int8, torch.bool]


@pytest.mark.parametrize("dtype", BYTES, ids=str)
def test_other_types_of_one_byte_are_not_codes(calls, dtype):
    layer = _layer(fp8=True)
    del calls[:]
    with pytest.raises(TypeError):
        dr.Linear(Stand(128, 256, dtype=dtype), Stand(1, 2, dtype=F32))
    with pytest.raises(TypeError):
        layer.forward(Stand(5, 256, dtype=dtype), Stand(2, 5, dtype=F32), Stand(3, dtype=I32), out=Stand(5, 128))
    with pytest.raises(ValueError):
        dr.quant_rows(Stand(5, 256), Stand(5, 256, dtype=dtype), Stand(2, 5, dtype=F32))
    assert not calls


def test_codes_may_be_bytes(calls):
    layer = dr.Linear(Stand(128, 256, dtype=torch.uint8), Stand(1, 2, dtype=F32))
    codes, scales = dr.quant_rows(Stand(5, 256), Stand(5, 256, dtype=torch.uint8), Stand(2, 5, dtype=F32))
    layer.forward(codes, scales, out=Stand(5, 128))
    assert layer.fp8 and [c[0] for c in calls] == ["dr_linear_create", "dr_quant_rows", "dr_linear_forward"]


def test_a_product_that_autograd_would_follow_is_refused(calls):
    layer, off = _layer(), Stand(3, dtype=I32)
    x, trained = Stand(5, 256, requires_grad=True), dr.Linear(Stand(256, 256, requires_grad=True), n_groups=2)
    del calls[:]
    with pytest.raises(RuntimeError, match="no_grad"):
        layer.forward(x, None, off, out=Stand(5, 128))
    with pytest.raises(RuntimeError, match="no_grad"):
        trained(Stand(5, 256), None, off, out=Stand(5, 128))
    with pytest.raises(RuntimeError, match="no_grad"):
        dr.quant_rows(x, Stand(5, 256, dtype=E4M3), Stand(2, 5, dtype=F32))
    assert not calls
    with torch.no_grad():
        layer.forward(x, None, off, out=Stand(5, 128))
        trained(x, None, off, out=Stand(5, 128))
        dr.quant_rows(x, Stand(5, 256, dtype=E4M3), Stand(2, 5, dtype=F32))
    layer.wgrad(x, Stand(5, 128, requires_grad=True), off, out=Stand(256, 256, dtype=F32))  # (gradients are what is asked for)
    layer.dgrad(Stand(5, 128, requires_grad=True), off, out=Stand(5, 256))
    assert len(calls) == 5
