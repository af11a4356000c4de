"""Operators that compute with a rollout arena's linear weights: cases, inputs, plain forms and 64-bit values.

Four kinds of case:

* ``quant``   rows of activations -> e4m3 with one fp32 scale per row and 128 columns (plain, through SwiGLU, or gathered);
* ``linear``  y = x W^T with e4m3 operands, x scaled per row and 128 columns, W per 128 x 128 block;
* ``experts`` the same product for rows sorted by expert, ragged groups, e4m3 or bf16 weights;
* ``grads``   the gradients of the bf16 product by expert: dx = dy W, dW = dy^T x in fp32.

With ``own`` false the plain forms run (elementary torch operations in 32 bits), with ``own`` true the package's kernels.
"""
import math

import torch

own = False

MOST_FLOPS = 2.0 * 8192 * 24576 * 4096  # of the largest listed case; a drawn one costs no more
DEV = "cuda"


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a decode step entering a layer: hidden 4096
        dict(name="quant_token", op="quant", rows=1, cols=4096, x="bf16", form="plain"),
        # a prefill chunk between the two MLP products: SwiGLU of width 12288, quantised on the way
        dict(name="quant_swiglu_prefill", op="quant", rows=8192, cols=12288, x="bf16", form="swiglu"),
        # fused qkv of the 8B shape, one sequence decoding
        dict(name="linear_decode_1", op="linear", rows=1, n=6144, k=4096, y="bf16"),
        # gate and up of the 8B shape, a decode batch of 64
        dict(name="linear_decode_64", op="linear", rows=64, n=24576, k=4096, y="bf16"),
        # down of the tiny shape: a contraction that ends inside a scale block, an odd number of rows
        dict(name="linear_ragged", op="linear", rows=777, n=256, k=688, y="bf16"),
        # gate and up of the 8B shape over a prefill chunk
        dict(name="linear_prefill", op="linear", rows=8192, n=24576, k=4096, y="bf16"),
        # eight sequences decoding through 128 experts, eight for each token: mostly one row an expert
        dict(name="experts_fp8_decode", op="experts", type="fp8", tokens=8, top=8, experts=128, n=1536, k=2048, skew=1.0),
        # a prefill chunk through the same experts
        dict(name="experts_fp8_prefill", op="experts", type="fp8", tokens=4096, top=8, experts=128, n=1536, k=2048, skew=1.0),
        # bf16 down projection of the experts, a small decode batch
        dict(name="experts_bf16_decode", op="experts", type="bf16", tokens=16, top=8, experts=128, n=2048, k=768, skew=1.0),
        # bf16 gate and up of the experts, a training micro-batch
        dict(name="experts_bf16_train", op="experts", type="bf16", tokens=4096, top=8, experts=128, n=1536, k=2048, skew=0.5),
        # its gradients
        dict(name="grads_train", op="grads", tokens=4096, top=8, experts=128, n=1536, k=2048, skew=0.5),
        # gradients of a small layer whose router prefers a few experts: empty and odd groups
        dict(name="grads_skewed", op="grads", tokens=501, top=2, experts=8, n=384, k=512, skew=4.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A weight's dimension: a multiple of 16, log-uniform."""
    w = max(1, _log(rng, lo, hi) // 16) * 16
    return w + 16 if w == 3072 else w


def draw(rng):
    while True:
        op = rng.choice(["quant", "linear", "linear", "experts", "experts", "grads"])
        if op == "quant":
            form = rng.choice(["plain", "swiglu", "gather"])
            cols = _log(rng, 64, 12288)
            if rng.random() < 0.75:
                cols = max(8, cols // 8 * 8)
            c = dict(op=op, rows=_log(rng, 1, 8192), cols=cols, x=rng.choice(["bf16", "bf16", "f32"]), form=form)
        elif op == "linear":
            c = dict(op=op, rows=_log(rng, 1, 8192), n=_width(rng, 128, 24576), k=_width(rng, 128, 12288), y="bf16")
        else:
            experts = rng.choice([8, 16, 33, 64, 128])
            c = dict(op=op, tokens=_log(rng, 1, 4096), top=min(experts, rng.choice([1, 2, 4, 8])), experts=experts,
                     n=_width(rng, 128, 2048), k=_width(rng, 128, 2048), skew=rng.choice([0.0, 0.5, 1.0, 3.0]))
            if op == "experts":
                c["type"] = rng.choice(["fp8", "bf16"])
        if work(c)["flops"] <= MOST_FLOPS:
            return c


def work(case):
    if case["op"] == "quant":
        r, c = case["rows"], case["cols"]
        size = 2 if case["x"] == "bf16" else 4
        reads = r * c * size * (2 if case["form"] == "swiglu" else 1) + (8 * r if case["form"] == "gather" else 0)
        return {"bytes": reads + r * c + 4 * r * -(-c // 128), "flops": 4 * r * c}
    if case["op"] == "linear":
        m, n, k = case["rows"], case["n"], case["k"]
        kb = -(-k // 128)
        return {"bytes": m * k + 4 * m * kb + n * k + 4 * -(-n // 128) * kb + 2 * m * n, "flops": 2.0 * m * n * k}
    t, e, n, k = case["tokens"], case["experts"], case["n"], case["k"]
    m = t * case["top"]
    met = e * (1 - (1 - case["top"] / e) ** t)  # experts that at least one token goes to, were they all alike
    kb = -(-k // 128)
    if case["op"] == "experts":
        if case["type"] == "fp8":
            b = m * k + 4 * m * kb + met * n * (k + 4 * kb / 128) + 2 * m * n
        else:
            b = 2 * (m * k + met * n * k + m * n)
        return {"bytes": b + 4 * (e + 1), "flops": 2.0 * m * n * k}
    return {"bytes": 2 * (m * n + m * k + met * n * k + m * k) + 4 * e * n * k + 4 * (e + 1), "flops": 4.0 * m * n * k}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _activations(g, rows, cols):
    """What enters a linear layer: normal values, a few columns some twenty times as large."""
    x = torch.randn(rows, cols, device=DEV, generator=g)
    return x * (1 + 20 * (torch.rand(cols, device=DEV, generator=g) < 0.003))


def _by_rows(x):
    """(e4m3 codes, fp32 scales [column blocks, rows]) of each row's blocks of 128 columns."""
    rows, cols = x.shape
    kb = -(-cols // 128)
    p = torch.nn.functional.pad(x, (0, kb * 128 - cols)).view(rows, kb, 128)
    s = (p.abs().amax(2) / 448).clamp(2.0 ** -126, torch.finfo(torch.float32).max)
    q = (p / s[:, :, None]).to(torch.float8_e4m3fn).view(rows, kb * 128)[:, :cols]
    return q.contiguous(), s.t().contiguous()


def _by_blocks(w):
    """(e4m3 codes, fp32 scales) of a weight, one scale for each 128 x 128 block."""
    r, c = w.shape
    rb, cb = -(-r // 128), -(-c // 128)
    p = torch.nn.functional.pad(w, (0, cb * 128 - c, 0, rb * 128 - r)).view(rb, 128, cb, 128)
    s = (p.abs().amax((1, 3)) / 448).clamp(2.0 ** -126, torch.finfo(torch.float32).max)
    q = (p / s[:, None, :, None]).to(torch.float8_e4m3fn).view(rb * 128, cb * 128)[:r, :c]
    return q.contiguous(), s.contiguous()


def _route(g, tokens, top, experts, skew):
    """Where each expert's rows begin: every token goes to its `top` best of random scores, some experts liked more."""
    liked = skew * torch.randn(experts, device=DEV, generator=g)
    pick = (torch.randn(tokens, experts, device=DEV, generator=g) + liked).topk(top, dim=1).indices
    count = torch.zeros(experts, dtype=torch.int32, device=DEV).scatter_add_(
        0, pick.reshape(-1), torch.ones(tokens * top, dtype=torch.int32, device=DEV))
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = count.cumsum(0)
    return offsets, int(count.max())


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["op"] == "quant":
        rows, cols = case["rows"], case["cols"]
        source = 2 * rows + 3 if case["form"] == "gather" else rows
        x = _activations(g, source, 2 * cols if case["form"] == "swiglu" else cols)
        s["src"] = x if case["x"] == "f32" else x.bfloat16()
        s["index"] = torch.randint(source, (rows,), device=DEV, generator=g) if case["form"] == "gather" else None
        s["codes"] = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=DEV)
        s["scales"] = torch.empty(-(-cols // 128), rows, dtype=torch.float32, device=DEV)
        return s
    n, k = case["n"], case["k"]
    if case["op"] == "linear":
        rows, groups = case["rows"], 1
        s["offsets"], s["cap"] = None, rows
    else:
        rows, groups = case["tokens"] * case["top"], case["experts"]
        s["offsets"], s["cap"] = _route(g, case["tokens"], case["top"], groups, case["skew"])
    s["groups"] = groups
    x, w = _activations(g, rows, k), torch.randn(groups * n, k, device=DEV, generator=g) * 0.02
    if case["op"] == "linear" or case.get("type") == "fp8":
        s["src"], s["src_scale"] = _by_rows(x)
        s["weight"], s["weight_scale"] = _by_blocks(w)
    else:
        s["src"], s["src_scale"] = x.bfloat16(), None
        s["weight"], s["weight_scale"] = w.bfloat16(), None
    if case["op"] == "grads":
        s["dy"] = (torch.randn(rows, n, device=DEV, generator=g) * 1e-2).bfloat16()
        s["dx"] = torch.empty(rows, k, dtype=torch.bfloat16, device=DEV)
        s["dw"] = torch.empty(groups * n, k, dtype=torch.float32, device=DEV)
    else:
        s["out"] = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV)
    if own:
        import paper_2607_22614_b200 as dr
        s["layer"] = dr.Linear(s["weight"], s["weight_scale"], n_groups=groups)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    if s["op"] == "quant":
        import paper_2607_22614_b200 as dr
        return dr.quant_rows(s["src"], s["codes"], s["scales"], row_index=s["index"], swiglu=s["form"] == "swiglu")
    if s["op"] == "grads":
        return (s["layer"].dgrad(s["dy"], s["offsets"], out=s["dx"]),
                s["layer"].wgrad(s["src"], s["dy"], s["offsets"], out=s["dw"]))
    return s["layer"].forward(s["src"], s["src_scale"], s["offsets"], out=s["out"])


def _wide_rows(q, scale):
    """Codes times their row scales, in 32 bits."""
    return q.float() * scale.t().repeat_interleave(128, dim=1)[:, :q.shape[1]]


def _wide_blocks(q, scale):
    return q.float() * scale.repeat_interleave(128, dim=0)[:q.shape[0]].repeat_interleave(128, dim=1)[:, :q.shape[1]]


def _padded(s, v):
    """Rows sorted by expert -> [experts, largest group, columns], zeros behind each group's rows."""
    at = s["offsets"][:-1, None] + torch.arange(s["cap"], device=DEV)
    inside = at < s["offsets"][1:, None]
    return torch.where(inside[:, :, None], v[torch.where(inside, at, 0).long()], 0)


def _ragged(s, v):
    """The way back: [experts, largest group, columns] -> rows sorted by expert."""
    row = torch.arange(s["src"].shape[0], device=DEV)
    e = torch.searchsorted(s["offsets"][1:], row, right=True)
    return v[e, row - s["offsets"][e]]


def _plain(s):
    if s["op"] == "quant":
        x = s["src"].float()
        if s["index"] is not None:
            x = x[s["index"]]
        if s["form"] == "swiglu":
            gate, up = x.chunk(2, dim=1)
            x = gate / (1 + torch.exp(-gate)) * up
        return _by_rows(x)
    if s["weight_scale"] is None:
        x, w = s["src"].float(), s["weight"].float()
    else:
        x, w = _wide_rows(s["src"], s["src_scale"]), _wide_blocks(s["weight"], s["weight_scale"])
    if s["op"] == "linear":
        return (x @ w.t()).bfloat16()
    w = w.view(s["groups"], s["n"], s["k"])
    x = _padded(s, x)
    if s["op"] == "experts":
        return _ragged(s, torch.bmm(x, w.transpose(1, 2))).bfloat16()
    dy = _padded(s, s["dy"].float())
    return _ragged(s, torch.bmm(dy, w)).bfloat16(), torch.bmm(dy.transpose(1, 2), x).view(-1, s["k"])


# ---- the values in 64 bits -----------------------------------------------------------------------------------------
def _nearest_e4m3(v):
    """v rounded to the nearest e4m3 value, ties to the even one, magnitudes above 448 held there."""
    a = v.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(v) * torch.round(a / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quant":
        codes, scales = [], []
        for at in range(0, case["rows"], 1024):
            x = (s["src"][at:at + 1024] if s["index"] is None else s["src"][s["index"][at:at + 1024]]).double()
            if case["form"] == "swiglu":
                gate, up = x[:, :case["cols"]], x[:, case["cols"]:]
                x = gate * torch.sigmoid(gate) * up
            parts, sc = [], []
            for c in range(0, case["cols"], 128):
                b = x[:, c:c + 128]
                m = (b.abs().max(dim=1).values / 448).clamp(2.0 ** -126, torch.finfo(torch.float32).max)
                parts.append(_nearest_e4m3(b / m[:, None]).to(torch.float32))  # an e4m3 value is exact in 32 bits
                sc.append(m)
            codes.append(torch.cat(parts, dim=1))
            scales.append(torch.stack(sc))
        return torch.cat(codes), torch.cat(scales, dim=1)
    n, k, groups = case["n"], case["k"], s["groups"]
    ends = [0, case["rows"]] if s["offsets"] is None else s["offsets"].tolist()
    fp8 = s["weight_scale"] is not None
    rows = ends[-1]
    y = torch.zeros(rows, k if case["op"] == "grads" else n, dtype=torch.float64, device=DEV)
    dw = torch.zeros(groups * n, k, dtype=torch.float64, device=DEV) if case["op"] == "grads" else None
    for e in range(groups):
        lo, hi = ends[e], ends[e + 1]
        if lo == hi:
            continue
        w = s["weight"][e * n:(e + 1) * n].double()
        x = s["src"][lo:hi].double()
        if case["op"] == "grads":
            d = s["dy"][lo:hi].double()
            y[lo:hi] = d @ w
            dw[e * n:(e + 1) * n] = d.t() @ x
        elif not fp8:
            y[lo:hi] = x @ w.t()
        else:
            block = torch.arange(e * n, (e + 1) * n, device=DEV) // 128
            for b in range(-(-k // 128)):
                part = x[:, 128 * b:128 * b + 128] @ w[:, 128 * b:128 * b + 128].t()
                y[lo:hi] += part * s["src_scale"][b, lo:hi].double()[:, None] * s["weight_scale"][block, b].double()[None, :]
    return y if dw is None else (y, dw)
