"""Plain 64-bit forms of the linear layers' operators, and the error bounds that their tests allow."""
import torch

DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def e4m3_nearest(v):
    """float64 -> the nearest e4m3 value, ties to even, saturating."""
    a = v.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign(torch.round(a / step) * step, v)


def blocks_of(rows, cols):
    return -(-rows // 128), -(-cols // 128)


def quant_weight(w):
    """float32 [rows, cols] -> e4m3 codes and block scales (any valid pair does: the product is tested on codes and scales)."""
    r, c = w.shape
    rb, cb = blocks_of(r, c)
    p = torch.nn.functional.pad(w, (0, cb * 128 - c, 0, rb * 128 - r)).view(rb, 128, cb, 128)
    s = (p.abs().amax((1, 3)) / 448).clamp(min=2.0 ** -126)
    q = (p / s[:, None, :, None]).to(torch.float8_e4m3fn).view(rb * 128, cb * 128)[:r, :c]
    return q.contiguous(), s.contiguous()


def wide_weight(q, s):
    return q.double() * s.double().repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]


def wide_rows(q, s):
    return q.double() * s.double().t().repeat_interleave(128, 1)[:q.shape[0], :q.shape[1]]


def product(a, b, out_dtype):
    """a @ b in 64 bits and the allowed error of an fp32 accumulation of it in any order, rounded to out_dtype.

    n products, each exact in fp32 or rounded once (2^-24), summed in fp32 with at most one rounding or truncation (2^-23) per
    addition: the error is below (n + 3) 2^-23 sum |a||b|.  Rounding the result to nearest adds up to half a unit in the last
    place: 2^-p of the result with p significant bits, 8 in bf16 and 24 in fp32."""
    y = a @ b
    mass = a.abs() @ b.abs()
    n = a.shape[1]
    unit = 2.0 ** -8 if out_dtype == torch.bfloat16 else 2.0 ** -24
    sums = (n + 3) * 2.0 ** -23 * mass
    return y, sums + unit * (y.abs() + sums) + 1e-40


def check(got, want, tol, what=""):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, first {bad.nonzero()[0].tolist()}: " \
        f"{got[tuple(bad.nonzero()[0])].item()} for {want[tuple(bad.nonzero()[0])].item()}"


def offsets_of(sizes, lead=0):
    o = torch.zeros(len(sizes) + 1, dtype=torch.int32)
    o[0] = lead
    o[1:] = lead + torch.tensor(sizes, dtype=torch.int32).cumsum(0)
    return o.to(DEV), [int(v) for v in o]


def strided(rows, cols, dtype, pad, shift=0, fill=0.0):
    """A rows x cols view with `pad` spare elements behind each row and `shift` before the first, and its whole buffer."""
    buf = torch.full((shift + rows * (cols + pad) + 64,), fill, device=DEV).to(dtype)
    return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], buf
