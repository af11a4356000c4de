"""Operators of the attention path over a rollout's 8-bit key and value cache: cases, inputs, plain forms and 64-bit values.

Three kinds of case:

* ``extend``  block tables, positions and the runs of cache slots that new rows go to, from request lengths (integers);
* ``heads``   norms of queries and keys for each head with the position rotation: ``forward`` (training), ``append`` (rollout: keys and
              values go into the cache) and ``grads``;
* ``attend``  attention over the cache: single tokens, a few drafted ones, prompts; grouped heads, ragged lengths, windows with sinks.

The cache holds e4m3 codes [blocks, kv heads, block tokens, head dim], and for each block and head one scale, a power of two: the
smallest for which every value of the block is within 448 scales.

With ``own`` false the plain forms run (elementary torch operations), with ``own`` true the package's kernels.
"""
import math

import torch

own = False

DEV = "cuda"
EPS, BASE = 1e-6, 1e6
LEAST = 2.0 ** -100  # of scales
MOST_FLOPS, MOST_BYTES = 5.9e11, 1.1e9  # of the largest listed cases; a drawn one costs no more
MOST_PAIRS = 2 * 32 * 4900 * 9100  # scores of the plain form in memory at once


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a decode step of 64 sequences: every 64th token needs a block, two sequences end, one idles
        dict(name="extend_decode", op="extend", requests=64, block=64, longest=32768, kind="decode"),
        # 200 prompts admitted at once
        dict(name="extend_prompts", op="extend", requests=200, block=64, longest=300, kind="prompts"),
        # one token of the 8B shape between its qkv product and its attention
        dict(name="heads_token", op="heads", form="append", q=32, kv=8, dim=128, block=64, requests=1, least=1, most=1, x="bf16"),
        # a prefill chunk of the 8B shape on its way into the cache: two prompts of odd lengths
        dict(name="heads_prompts", op="heads", form="append", q=32, kv=8, dim=128, block=64, requests=2, least=3501, most=4691, x="bf16"),
        # a training micro-batch of the 8B shape
        dict(name="heads_train", op="heads", form="forward", q=32, kv=8, dim=128, rows=8192, x="bf16"),
        # its gradients
        dict(name="heads_grads", op="heads", form="grads", q=32, kv=8, dim=128, rows=8192, x="bf16"),
        # one sequence of the tiny shape at its start
        dict(name="attend_token", op="attend", q=4, kv=2, dim=64, block=16, requests=1, least=300, most=300, new="1", window=0, sinks=0),
        # a decode step of the 8B shape: 64 sequences of ragged lengths
        dict(name="attend_decode", op="attend", q=32, kv=8, dim=128, block=64, requests=64, least=700, most=32768, new="1", window=0,
             sinks=0),
        # one long sequence of the 30B-A3B shape
        dict(name="attend_long", op="attend", q=32, kv=4, dim=128, block=64, requests=1, least=131000, most=131000, new="1", window=0,
             sinks=0),
        # sequences of the 14B shape (one of four ranks) that see their last 1000 tokens and the first four
        dict(name="attend_window", op="attend", q=10, kv=2, dim=128, block=32, requests=32, least=500, most=20000, new="1", window=1000,
             sinks=4),
        # drafted tokens of the 8B shape, five a sequence, before they are verified
        dict(name="attend_drafts", op="attend", q=32, kv=8, dim=128, block=64, requests=16, least=900, most=9000, new="5", window=0,
             sinks=0),
        # prompts of the 8B shape, one of them behind a prefix that the cache holds already
        dict(name="attend_prompts", op="attend", q=32, kv=8, dim=128, block=64, requests=2, least=3501, most=9001, new="prompts",
             window=0, sinks=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["extend", "heads", "heads", "attend", "attend", "attend"])
        q, kv, dim = rng.choice([(32, 8, 128), (16, 8, 128), (40, 8, 128), (10, 2, 128), (32, 4, 128), (4, 2, 64), (16, 8, 64), (8, 1, 128)])
        block = rng.choice([16, 32, 64, 128])
        if op == "extend":
            kind = rng.choice(["decode", "prompts"])
            c = dict(op=op, requests=_log(rng, 1, 1000 if kind == "decode" else 200), block=block,
                     longest=_log(rng, 2, 32768 if kind == "decode" else 300), kind=kind)
        elif op == "heads":
            form = rng.choice(["append", "forward", "grads"])
            c = dict(op=op, form=form, q=q, kv=kv, dim=dim, x=rng.choice(["bf16", "bf16", "f32"]))
            if form == "append":
                requests = _log(rng, 1, 64)
                most = 1 if rng.random() < 0.4 else _log(rng, 1, 8192 / requests)
                c.update(block=block, requests=requests, least=max(1, most // 3), most=most)
            else:
                c.update(rows=_log(rng, 1, 8192))
            if c["x"] == "f32" and 4096 * 6144 < q * dim * (c.get("rows") or c["requests"] * c["most"]):
                continue
        else:
            new = rng.choice(["1", "1", str(rng.randint(2, 8)), "prompts"])
            requests = _log(rng, 1, 8 if new == "prompts" else 64)
            most = _log(rng, 64, 9000 if new == "prompts" else 32768)
            windowed = rng.random() < 0.3
            c = dict(op=op, q=q, kv=kv, dim=dim, block=block, requests=requests, least=max(8, _log(rng, most / 16, most)), most=most,
                     new=new, window=_log(rng, 16, 4096) if windowed else 0, sinks=rng.choice([0, 1, 4, 70]) if windowed else 0)
            c["most"] = max(c["most"], c["least"])
            lens, added = _lengths(c)
            if requests * q * max(added) * max(lens) > MOST_PAIRS:
                continue
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, even over their logarithm, in no order."""
    if n == 1:
        return [hi]
    at = sorted(range(n), key=lambda i: (i * 0.6180339887) % 1.0)
    return [int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in at]


def _lengths(case):
    """Tokens that the cache holds for each request, the new ones among them, and how many of them are new."""
    lens = _spread(case["least"], case["most"], case["requests"])
    if case["new"] == "prompts":  # every other one has a prefix that was there before
        return lens, [n if i % 2 == 0 else max(1, n // 2) for i, n in enumerate(lens)]
    return lens, [min(n, int(case["new"])) for n in lens]


def _seen(length, added, window, sinks):
    """Pairs of a new token and a token that it sees."""
    total = 0
    first = length - added
    if window == 0:
        return added * first + added * (added + 1) // 2
    for p in range(first, length):
        far = max(0, p + 1 - window)
        total += p + 1 - far + min(far, sinks)
    return total


def _added(case):
    """What arrives for each request of an extend case: (tokens held, tokens arriving; -1: the request ends)."""
    n = case["requests"]
    lens = _spread(1, case["longest"], n)
    if case["kind"] == "prompts":
        return [0] * n, lens
    return lens, [(-1 if i % 32 == 7 else 0 if i % 64 == 9 else 1) for i in range(n)]


def work(case):
    if case["op"] == "extend":
        held, added = _added(case)
        b, rows = case["block"], sum(max(0, a) for a in added)
        new = sum(-(-(h + a) // b) - -(-h // b) for h, a in zip(held, added) if a > 0)
        back = sum(-(-h // b) for h, a in zip(held, added) if a < 0)
        n_runs = min(rows, rows // b + 2 * case["requests"])
        return {"bytes": 4.0 * (2 * len(held) + 2 * new + 2 * back + len(held) + 1 + rows + 4 * n_runs + len(held) + 4), "flops": 0.0}
    q, kv, dim = case["q"], case["kv"], case["dim"]
    if case["op"] == "heads":
        size = 2 if case["x"] == "bf16" else 4
        if case["form"] == "append":
            rows = sum(_spread(case["least"], case["most"], case["requests"]))
            return {"bytes": float(rows * dim * (size * (2 * q + 2 * kv) + 2 * kv) + 4 * rows), "flops": 10.0 * rows * (q + kv) * dim}
        rows, heads = case["rows"], q + kv
        passes = 2 if case["form"] == "forward" else 3
        return {"bytes": float(passes * size * rows * heads * dim + 4 * rows), "flops": (10.0 if passes == 2 else 20.0) * rows * heads * dim}
    lens, added = _lengths(case)
    pairs = sum(_seen(n, a, case["window"], case["sinks"]) for n, a in zip(lens, added))
    read = sum(n if case["window"] == 0 else min(n, case["window"] + a - 1 + case["sinks"]) for n, a in zip(lens, added))
    rows, b = sum(added), case["block"]
    return {"bytes": float(2 * read * kv * dim + 8 * -(-read // b) * kv + 4 * -(-read // b) + 4 * rows * q * dim),
            "flops": 4.0 * pairs * q * dim}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _scale_of(most):
    """The power of two for blocks whose largest magnitudes are `most` (64 bits)."""
    f, e = torch.frexp(most.double() / 448)
    return torch.exp2(torch.where(f > 0.5, e, e - 1).double()).clamp(min=LEAST).where(most > 0, torch.full_like(most, LEAST).double()).float()


def _cache(g, blocks, kv, block, dim, size):
    """Codes and scales of a cache whose blocks hold normal values, some heads larger than others."""
    codes = torch.empty(blocks, kv, block, dim, dtype=torch.float8_e4m3fn, device=DEV)
    scales = torch.empty(blocks, kv, device=DEV)
    step = max(1, (1 << 28) // (kv * block * dim))
    for at in range(0, blocks, step):
        x = torch.randn(min(step, blocks - at), kv, block, dim, device=DEV, generator=g)
        x *= size * torch.exp2(torch.randn(1, kv, 1, dim, device=DEV, generator=g) * 0.5)
        s = _scale_of(x.abs().amax((2, 3)))
        codes[at:at + step] = (x / s[:, :, None, None]).to(torch.float8_e4m3fn)
        scales[at:at + step] = s
    return codes, scales


def _table(g, lens, block, spare=0):
    """A block table over scattered blocks, and how many blocks the cache has."""
    need = [-(-n // block) for n in lens]
    width, total = max(need) + spare, sum(need)
    order = torch.randperm(total + 5, device=DEV, generator=g).int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, total + 5


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["op"] == "extend":
        held, added = _added(case)
        b = case["block"]
        most = max(-(-(h + max(a, 0)) // b) for h, a in zip(held, added))
        s["table"], blocks = _table(g, [max(h, 1) for h in held], b, most + 1 - max(-(-max(h, 1) // b) for h in held))
        taken = sum(-(-max(h, 1) // b) for h in held)
        more = sum(-(-(h + a) // b) - -(-h // b) for h, a in zip(held, added) if a > 0)
        s["blocks"] = blocks + more
        s["free"] = torch.zeros(s["blocks"], dtype=torch.int32, device=DEV)
        s["free"][:s["blocks"] - taken] = taken + torch.randperm(s["blocks"] - taken, device=DEV, generator=g).int()
        s["state"] = _ints([s["blocks"] - taken, 0])
        s["held"], s["added"] = _ints(held), _ints(added)
        s["rows"] = sum(max(a, 0) for a in added)
        s["lengths_out"], s["state_out"] = torch.empty_like(s["held"]), torch.empty_like(s["state"])
        n_runs = min(s["rows"], s["rows"] // b + 2 * len(held))
        s["offsets"] = torch.empty(len(held) + 1, dtype=torch.int32, device=DEV)
        s["positions"] = torch.empty(s["rows"], dtype=torch.int32, device=DEV)
        s["runs"] = torch.empty(n_runs, 4, dtype=torch.int32, device=DEV)
        kv = torch.zeros(s["blocks"], 1, b, 64, dtype=torch.float8_e4m3fn, device=DEV), torch.ones(s["blocks"], 1, device=DEV)
        if own:
            import paper_2607_22614_b200 as dr
            s["cache"] = dr.KVCache(kv[0], kv[0].clone(), kv[1], kv[1].clone())
        return s
    q, kv, dim = case["q"], case["kv"], case["dim"]
    if case["op"] == "heads":
        _prepare_heads(case, g, s)
    else:
        lens, added = _lengths(case)
        s["table"], blocks = _table(g, lens, case["block"])
        s["k"], s["k_scale"] = _cache(g, blocks, kv, case["block"], dim, 1.0)
        s["v"], s["v_scale"] = _cache(g, blocks, kv, case["block"], dim, 0.5)
        offsets = [0]
        for a in added:
            offsets.append(offsets[-1] + a)
        s["lengths"], s["offsets"] = _ints(lens), None if case["new"] == "1" else _ints(offsets)
        # queries lie in the rows of a qkv product's output
        s["queries"] = (1.5 * torch.randn(offsets[-1], (q + 2 * kv) * dim, device=DEV, generator=g)).bfloat16()[:, :q * dim]
        s["out"] = torch.empty(offsets[-1], q * dim, dtype=torch.bfloat16, device=DEV)
        s["cap"], s["cap_new"] = max(lens), max(added)
    if own:
        import paper_2607_22614_b200 as dr
        if "k" in s:
            s["cache"] = dr.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if case["op"] == "heads":
            s["heads"] = dr.QKHeads(q, kv, dim, s["q_norm"], s["k_norm"], base=BASE, eps=EPS)
    return s


def _prepare_heads(case, g, s):
    q, kv, dim = case["q"], case["kv"], case["dim"]
    kind = torch.bfloat16 if case["x"] == "bf16" else torch.float32
    s["q_norm"] = (1 + 0.3 * torch.randn(dim, device=DEV, generator=g)).to(kind)
    s["k_norm"] = (1 + 0.3 * torch.randn(dim, device=DEV, generator=g)).to(kind)
    if case["form"] == "append":
        added = _spread(case["least"], case["most"], case["requests"])
        b, n = case["block"], len(added)
        # a sequence at its start, one that ends inside a block, one that has just filled it
        held = [(0, b // 2 + 1, 3 * b)[i % 3] if case["most"] > 1 else (b // 2 + 1 + i % b) for i in range(n)]
        s["table"], blocks = _table(g, [h + a for h, a in zip(held, added)], b)
        s["k"], s["k_scale"] = _cache(g, blocks, kv, b, dim, 1.0)
        s["v"], s["v_scale"] = _cache(g, blocks, kv, b, dim, 0.5)
        runs, pos, row, table = [], [], 0, s["table"].tolist()
        for r in range(n):
            at, end = held[r], held[r] + added[r]
            pos += range(at, end)
            while at < end:
                m = min(b - at % b, end - at)
                runs.append([table[r][at // b], at % b, row, m])
                at, row = at + m, row + m
        s["runs"], s["positions"], rows = _ints(runs), _ints(pos), row
        s["out"] = torch.empty(rows, q * dim, dtype=kind, device=DEV)
    else:
        rows = case["rows"]
        # packed sequences, the later ones far into a long context
        i = torch.arange(rows, device=DEV)
        s["positions"] = torch.where(i < rows // 2, i, 100000 + i - rows // 2).int()
    s["x"] = torch.randn(rows, (q + 2 * kv) * dim, device=DEV, generator=g).mul_(1.7).to(kind)
    if case["form"] == "forward":
        s["out"] = torch.empty(rows, (q + kv) * dim, dtype=kind, device=DEV)
    if case["form"] == "grads":
        s["dy"] = (torch.randn(rows, (q + kv) * dim, device=DEV, generator=g) * 1e-2).to(kind)
        s["dx"] = torch.empty(rows, (q + kv) * dim, dtype=kind, device=DEV)
        s["dq_norm"], s["dk_norm"] = torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    if s["op"] == "extend":
        s["cache"].extend(s["added"], s["held"], s["table"], s["free"], s["state"], s["rows"], lengths_out=s["lengths_out"],
                          state_out=s["state_out"], offsets=s["offsets"], positions=s["positions"], runs=s["runs"])
        return s["offsets"], s["positions"], s["runs"], s["lengths_out"], s["state_out"], s["table"], s["free"]
    if s["op"] == "attend":
        return s["cache"].attend(s["queries"], s["lengths"], s["table"], s["offsets"], window=s["window"], sinks=s["sinks"], out=s["out"])
    if s["form"] == "forward":
        return s["heads"].forward(s["x"], s["positions"], out=s["out"])
    if s["form"] == "grads":
        return s["heads"].grad(s["x"], s["positions"], s["dy"], dx=s["dx"], dq_norm=s["dq_norm"], dk_norm=s["dk_norm"])
    s["heads"].append(s["x"], s["positions"], s["runs"], s["cache"], out=s["out"])
    return s["out"], s["k"], s["v"], s["k_scale"], s["v_scale"]


def _plain(s):
    if s["op"] == "extend":
        return _plain_extend(s)
    if s["op"] == "attend":
        return _plain_attend(s)
    q, kv, dim = s["q"], s["kv"], s["dim"]
    if s["form"] == "grads":
        return _plain_grads(s)
    x = s["x"][:, :(q + kv) * dim].float().view(-1, q + kv, dim)
    y = _rotate(_normed(x, _weights(s)), *_angles(s))
    if s["form"] == "forward":
        return y.reshape(x.shape[0], -1).to(s["x"].dtype)
    v = s["x"][:, (q + kv) * dim:].float().view(-1, kv, dim)
    _store(s["runs"], y[:, q:], s["k"], s["k_scale"])
    _store(s["runs"], v, s["v"], s["v_scale"])
    return y[:, :q].reshape(x.shape[0], -1).to(s["x"].dtype), s["k"], s["v"], s["k_scale"], s["v_scale"]


# ---- plain forms: heads
def _weights(s):
    """The norm's weight for each head."""
    return torch.cat([s["q_norm"].float().expand(s["q"], -1), s["k_norm"].float().expand(s["kv"], -1)])


def _angles(s):
    i = torch.arange(s["dim"] // 2, device=DEV, dtype=torch.float64)
    a = s["positions"].double()[:, None] * BASE ** (-2 * i / s["dim"])
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _normed(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _rotate(y, cos, sin):
    a, b = y.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _store(runs, values, codes, scales):
    """Rows of `values` [rows, heads, dim] into the cache, run by run: all of a run's block is written anew where its scale grows."""
    block, start, row, count = (runs[:, i].long() for i in range(4))
    j = torch.arange(codes.shape[2], device=DEV)
    fresh = (j >= start[:, None]) & (j < (start + count)[:, None])
    at = torch.where(fresh, row[:, None] + j - start[:, None], 0)
    new = values[at].permute(0, 2, 1, 3) * fresh[:, None, :, None]
    kept = (j < start[:, None])[:, None, :, None]
    was = torch.where(start[:, None] > 0, scales[block], torch.full_like(scales[block], LEAST))
    scale = torch.maximum(_scale_of(new.abs().amax((2, 3))), was)
    held = codes[block]
    wide = torch.where(kept, held.float() * was[:, :, None, None], new) / scale[:, :, None, None]
    codes[block] = torch.where(kept | fresh[:, None, :, None], wide, held.float()).to(torch.float8_e4m3fn)
    scales[block] = scale


def _plain_grads(s):
    q, kv, dim = s["q"], s["kv"], s["dim"]
    x = s["x"][:, :(q + kv) * dim].float().view(-1, q + kv, dim)
    cos, sin = _angles(s)
    g = _rotate(s["dy"].float().view(-1, q + kv, dim), cos, -sin)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    h = g * _weights(s)
    dx = r * (h - n * (h * n).mean(-1, keepdim=True))
    dw = (g * n).double().sum(0)
    return dx.reshape(x.shape[0], -1).to(s["x"].dtype), dw[:q].sum(0).float(), dw[q:].sum(0).float()


# ---- plain forms: block tables
def _plain_extend(s):
    b, rows = s["block"], s["rows"]
    held, added, table, free = s["held"].long(), s["added"].long(), s["table"], s["free"]
    count, width = s["state"][0].long(), table.shape[1]
    ends, new = added < 0, added.clamp(min=0)
    has = (held + b - 1) // b
    back = torch.where(ends, has, 0)
    column = torch.arange(width, device=DEV)
    place = torch.where(column < back[:, None], count + (back.cumsum(0) - back)[:, None] + column, free.numel())
    listed = torch.cat([free, free[:1]]).scatter(0, place.clamp(max=free.numel()).reshape(-1), table.reshape(-1))[:-1]
    available = count + back.sum()
    offsets = torch.cat([new.new_zeros(1), new.cumsum(0)])
    after = (held + new + b - 1) // b
    fits = (after <= width) & (offsets[1:] <= rows)
    want = torch.where((new > 0) & fits, after - has, 0)
    taken = want.cumsum(0)
    served = (new > 0) & fits & ((want == 0) | (taken <= available))
    fill = served[:, None] & (column >= has[:, None]) & (column < after[:, None])
    at = available - 1 - ((taken - want)[:, None] + column - has[:, None])
    table.copy_(torch.where(fill, listed[at.clamp(0, listed.numel() - 1)], table))
    lengths = torch.where(ends, 0, torch.where(served, held + new, held))
    row = torch.arange(rows, device=DEV)
    r = torch.searchsorted(offsets[1:], row, right=True).clamp(max=held.numel() - 1)
    positions = torch.where((row < offsets[-1]) & served[r], held[r] + row - offsets[r], -1)
    # runs: where a row is the first of its request or of a block
    first = (positions >= 0) & ((row == offsets[r]) | (positions % b == 0))
    index = torch.where(first, first.long().cumsum(0) - 1, s["runs"].shape[0])
    n = torch.minimum(b - positions % b, offsets[r + 1] - row)
    entry = torch.stack([table[r, (positions // b).clamp(0, width - 1)].long(), positions % b, row, n], dim=1)
    runs = torch.tensor([-1, 0, 0, 0], device=DEV).repeat(s["runs"].shape[0] + 1, 1)
    runs[index] = torch.where(first[:, None], entry, runs[-1])
    free.copy_(listed)
    state = torch.stack([available - torch.where(served, want, 0).sum(), ((new > 0) & ~served).sum()])
    return offsets.int(), positions.int(), runs[:-1].int(), lengths.int(), state.int(), table, free


# ---- plain forms: attention
def _plain_attend(s):
    q, kv, dim, b = s["q"], s["kv"], s["dim"], s["block"]
    n_req, cap, new, group = s["requests"], s["cap"], s["cap_new"], q // kv
    lens = s["lengths"].long()
    offsets = torch.arange(n_req + 1, device=DEV) if s["offsets"] is None else s["offsets"].long()
    added = offsets[1:] - offsets[:-1]
    t = torch.arange(cap, device=DEV)
    block = s["table"][:, t // b].long().clamp(min=0)  # [requests, tokens]
    held = (t < lens[:, None])[:, None, :, None]

    def wide(codes, scales):  # [requests, heads, tokens, dim]
        x = codes[block, :, t % b].float().mul_(scales[block][..., None]).permute(0, 2, 1, 3)
        return torch.where(held, x, 0)

    i = torch.arange(new, device=DEV)
    mine = i < added[:, None]
    rows = torch.where(mine, offsets[:-1, None] + i, 0)
    x = s["queries"][rows].float().view(n_req, new, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(n_req, kv, new * group, dim)
    p = (lens - added)[:, None] + i  # positions of the new tokens
    seen = (t <= p[..., None]) & (t < lens[:, None, None]) & mine[..., None]
    if s["window"]:
        seen &= (t > p[..., None] - s["window"]) | (t < s["sinks"])
    seen = seen[:, None, :, None, :]
    score = torch.matmul(x, wide(s["k"], s["k_scale"]).transpose(2, 3)).mul_(dim ** -0.5).view(n_req, kv, new, group, cap)
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = score.sum(-1, keepdim=True)
    y = torch.matmul(score.view(n_req, kv, new * group, cap), wide(s["v"], s["v_scale"])).view(n_req, kv, new, group, dim)
    y = torch.where(total > 0, y / total, 0).permute(0, 2, 1, 3, 4).reshape(n_req, new, q * dim)
    s["out"][rows[mine]] = y[mine].to(s["out"].dtype)
    return s["out"]


# ---- the values in 64 bits -----------------------------------------------------------------------------------------
def _nearest_e4m3(v):
    """v rounded to the nearest e4m3 value, ties to the even one, magnitudes above 448 held there."""
    a = v.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(v) * torch.round(a / step) * step


def exact(case, seed):
    if case["op"] == "extend":
        return None  # whole numbers
    s = prepare(case, seed)
    return _exact_attend(s) if case["op"] == "attend" else _exact_heads(s)


def _exact_heads(s):
    q, kv, dim = s["q"], s["kv"], s["dim"]
    half, rows = dim // 2, s["x"].shape[0]
    freq = torch.tensor([BASE ** (-2.0 * i / dim) for i in range(half)], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones(rows, half, dtype=torch.float64, device=DEV), s["positions"].double()[:, None] * freq)
    out = torch.empty(rows, (q + kv) * dim, dtype=torch.float64, device=DEV)
    dw = torch.zeros(2, dim, dtype=torch.float64, device=DEV)
    for h in range(q + kv):
        x = s["x"][:, h * dim:(h + 1) * dim].double()
        w = (s["q_norm"] if h < q else s["k_norm"]).double()
        size = (x.square().sum(1, keepdim=True) / dim + EPS).sqrt()
        if s["form"] == "grads":
            d = s["dy"][:, h * dim:(h + 1) * dim].double()
            back = torch.complex(d[:, :half], d[:, half:]) * turn.conj()
            g = torch.cat([back.real, back.imag], dim=1)
            dw[int(h >= q)] += (g * x / size).sum(0)
            out[:, h * dim:(h + 1) * dim] = g * w / size - x * (g * w * x).sum(1, keepdim=True) / (dim * size ** 3)
        else:
            y = x / size * w
            z = torch.complex(y[:, :half], y[:, half:]) * turn
            out[:, h * dim:(h + 1) * dim] = torch.cat([z.real, z.imag], dim=1)
    if s["form"] == "forward":
        return out
    if s["form"] == "grads":
        return out, dw[0], dw[1]
    values = {"k": out[:, q * dim:].view(rows, kv, dim), "v": s["x"][:, (q + kv) * dim:].double().view(rows, kv, dim)}
    codes = {c: s[c].float() for c in "kv"}
    scales = {c: s[c + "_scale"].double() for c in "kv"}
    for block, start, row, n in s["runs"].tolist():
        for c in "kv":
            new = values[c][row:row + n].transpose(0, 1)  # [heads, tokens, dim]
            most = new.abs().amax((1, 2))
            e = torch.ceil(torch.log2(most / 448))
            e = torch.where(448 * torch.exp2(e) < most, e + 1, e)
            e = torch.where(448 * torch.exp2(e - 1) >= most, e - 1, e)
            scale = torch.exp2(e).clamp(min=LEAST)
            if start:
                was = scales[c][block]
                scale = torch.maximum(scale, was)
                codes[c][block, :, :start] = _nearest_e4m3(codes[c][block, :, :start].double() * (was / scale)[:, None, None]).float()
            codes[c][block, :, start:start + n] = _nearest_e4m3(new / scale[:, None, None]).float()
            scales[c][block] = scale
    return out[:, :q * dim], codes["k"], codes["v"], scales["k"], scales["v"]


def _exact_attend(s):
    q, kv, dim, b = s["q"], s["kv"], s["dim"], s["block"]
    group, out = q // kv, torch.zeros(s["queries"].shape[0], q * dim, dtype=torch.float64, device=DEV)
    offsets = list(range(s["requests"] + 1)) if s["offsets"] is None else s["offsets"].tolist()
    for r, n in enumerate(s["lengths"].tolist()):
        lo, hi = offsets[r], offsets[r + 1]
        ids = s["table"][r, :-(-n // b)].long()
        pos = torch.arange(n - (hi - lo), n, device=DEV)[:, None]
        t = torch.arange(n, device=DEV)[None, :]
        hidden = t > pos
        if s["window"]:
            hidden |= (t <= pos - s["window"]) & (t >= s["sinks"])
        for h in range(kv):
            k = (s["k"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, dim)[:n]
            v = (s["v"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None]).reshape(-1, dim)[:n]
            for i in range(h * group, (h + 1) * group):
                x = s["queries"][lo:hi, i * dim:(i + 1) * dim].double() @ k.t() / math.sqrt(dim)
                out[lo:hi, i * dim:(i + 1) * dim] = torch.softmax(x.masked_fill(hidden, -math.inf), dim=1) @ v
    return out
