"""Plain 64-bit forms of the attention path's operators, and the error bounds that their tests allow."""
import math

import torch

from linear_util import DEV, e4m3_nearest, gen

E4M3 = torch.float8_e4m3fn
LEAST = 2.0 ** -100


# ---- block tables (plain Python) --------------------------------------------------------------------------------------
def extend(added, lengths, table, free, state, rows, block, n_blocks, n_runs):
    """One step as dr_kv_extend defines it: (offsets, positions, runs, lengths, table, free, state)."""
    lengths, table, free = list(lengths), [list(r) for r in table], list(free)
    width = len(table[0]) if table else 0
    lengths = [min(max(n, 0), width * block) for n in lengths]
    count = min(max(state[0], 0), n_blocks)
    for r, a in enumerate(added):
        if a < 0:
            for j in range(-(-lengths[r] // block)):
                if count < n_blocks:
                    free[count] = table[r][j]
                    count += 1
    offsets, positions, runs, refused, wanted, available = [0], [-1] * rows, [], 0, 0, count
    for r, a in enumerate(added):
        n, row, held = max(a, 0), offsets[-1], lengths[r]
        offsets.append(min(row + n, rows))
        if a < 0:
            lengths[r] = 0
        if n == 0:
            continue
        has = -(-held // block)
        fits = held + n <= width * block and row + n <= rows
        want = -(-(held + n) // block) - has if fits else 0
        wanted += want
        if not fits or (want and wanted > available):
            refused += 1
            continue
        for j in range(want):
            count -= 1
            table[r][has + j] = free[count]
        lengths[r] = held + n
        for i in range(n):
            positions[row + i] = held + i
        at, end = held, held + n
        while at < end:
            m = min(block - at % block, end - at)
            runs.append([table[r][at // block], at % block, row + at - held, m])
            at += m
    runs += [[-1, 0, 0, 0]] * (n_runs - len(runs))
    return offsets, positions, runs, lengths, table, free, [count, refused]


# ---- heads -----------------------------------------------------------------------------------------------------------
def rotation(positions, dim, base):
    i = torch.arange(dim // 2, dtype=torch.float64, device=positions.device)
    a = positions.double()[:, None] * base ** (-2 * i / dim)
    return torch.cos(a)[:, None], torch.sin(a)[:, None]


def heads(x, positions, n_q, n_kv, dim, q_norm, k_norm, base, eps):
    """Query and key heads of x, normed and rotated, in x's own (64-bit) type, differentiable."""
    y = x[:, :(n_q + n_kv) * dim].reshape(x.shape[0], n_q + n_kv, dim)
    if q_norm is not None:
        w = torch.cat([q_norm.expand(n_q, dim), k_norm.expand(n_kv, dim)])
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + eps) * w
    c, s = rotation(positions, dim, base)
    lo, hi = y.chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def scale_above(most):
    """The smallest power of two >= 2^-100 with most <= 448 scales."""
    s = torch.full_like(most, LEAST)
    e = torch.ceil(torch.log2(most.clamp(min=448 * LEAST) / 448))
    for d in (1, 0, -1):
        s = torch.where(448 * torch.exp2(e + d) >= most, torch.exp2(e + d), s)
    return s.clamp(min=LEAST)


def store(runs, values, codes, scales, block):
    """values [rows, heads, dim] in 64 bits into codes (as float64 values of codes) and scales, run by run."""
    for b, start, row, n in runs:
        if n == 0:
            continue
        new = values[row:row + n].transpose(0, 1)
        s = scale_above(new.abs().amax((1, 2)))
        if start:
            s = torch.maximum(s, scales[b])
            codes[b, :, :start] = e4m3_nearest(codes[b, :, :start] * (scales[b] / s)[:, None, None])
        codes[b, :, start:start + n] = e4m3_nearest(new / s[:, None, None])
        scales[b] = s


# ---- attention ---------------------------------------------------------------------------------------------------------
def make_cache(g, n_blocks, kv, block, dim, spread=2.0):
    """Codes and scales (powers of two) of normal values whose blocks differ in size."""
    out = []
    for _ in range(2):
        x = torch.randn(n_blocks, kv, block, dim, device=DEV, generator=g) * torch.exp2(spread * torch.randn(n_blocks, kv, 1, 1, device=DEV, generator=g))
        s = scale_above(x.double().abs().amax((2, 3))).float()
        out += [(x / s[:, :, None, None]).to(E4M3), s]
    return out[0], out[2], out[1], out[3]  # k, v, k_scale, v_scale


def make_table(g, lengths, block, n_blocks, width):
    need = [-(-n // block) for n in lengths]
    assert sum(need) <= n_blocks and max(need + [0]) <= width
    order = torch.randperm(n_blocks, device=DEV, generator=g).int()
    table = torch.full((len(lengths), width), -7, dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table


def attention(q, k, v, k_scale, v_scale, lengths, offsets, table, n_q, window=0, sinks=0, scale=None):
    """(out, allowed error) in 64 bits for the rows that requests own; NaN in the rows that none does.

    The allowed error, first order and doubled for the rest: a logit is off by delta = (dim + 4) 2^-23 of its sum of magnitudes (fp32 sums
    in any order, and three products) + 2^-17 max|q| sum|k| (a query may be split into codes relative to its largest value); each p by
    that, by 2^-11 (fp16), 2^-21 (exponential) and by 2^-36 of the largest (half a step of fp16 below 2^-14, where the largest is at
    least 2^11); sums of n by (n + 8) 2^-23; the result by 2^-8."""
    n_blocks, kv, block, dim = k.shape
    group, scale = n_q // kv, dim ** -0.5 if scale is None else scale
    out = torch.full((q.shape[0], n_q * dim), math.nan, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for r, n in enumerate(lengths):
        lo, hi = offsets[r], offsets[r + 1]
        if lo == hi:
            continue
        ids = table[r, :-(-n // block)].long()
        held = ((ids >= 0) & (ids < n_blocks)).repeat_interleave(block)[:n]
        ids = ids.clamp(0, n_blocks - 1)
        pos = torch.arange(n - (hi - lo), n, device=q.device)[:, None]
        t = torch.arange(n, device=q.device)[None]
        seen = (t <= pos) & held[None]
        if window:
            seen &= (t > pos - window) | (t < sinks)
        for h in range(n_q):
            c = h // group
            kk = (k[ids, c].double() * k_scale[ids, c].double()[:, None, None]).reshape(-1, dim)[:n]
            vv = (v[ids, c].double() * v_scale[ids, c].double()[:, None, None]).reshape(-1, dim)[:n]
            vv = torch.where(held[:, None], vv, 0)
            x = q[lo:hi, h * dim:(h + 1) * dim].double()
            s = torch.where(seen, scale * (x @ kk.t()), -math.inf)
            mass = abs(scale) * torch.where(seen, x.abs() @ kk.abs().t(), 0)
            rough = abs(scale) * x.abs().amax(1, keepdim=True) * torch.where(seen, kk.abs().sum(1)[None], 0)
            delta = ((dim + 4) * 2.0 ** -23 * mass + 2.0 ** -17 * rough).amax(1, keepdim=True) if n else 0
            p = torch.softmax(s, 1).nan_to_num(0.0) if not torch.isnan(s).any() else torch.softmax(s, 1)
            p = torch.where(seen.any(1, keepdim=True), p, 0)
            y = p @ vv
            size = p @ vv.abs()
            top = p.amax(1, keepdim=True) if n else torch.zeros(hi - lo, 1, dtype=torch.float64, device=q.device)
            every = torch.where(seen, 1.0, 0.0).double() @ vv.abs()
            rel = 2 * (2 * delta + 2.0 ** -11 + 2.0 ** -21 + (n + 8) * 2.0 ** -23)
            err = rel * size + 2.0 ** -36 * top * every
            out[lo:hi, h * dim:(h + 1) * dim] = y
            tol[lo:hi, h * dim:(h + 1) * dim] = err + 2.0 ** -8 * (y.abs() + err) + 1e-38
    return out, tol
