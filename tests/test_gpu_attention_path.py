"""The attention path's operators as they are used together: prompts, then tokens one by one, eager and captured, over an arena."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2607_22614_b200 as dr
from attend_util import attention
from linear_util import DEV, gen
from synth.configs import MID

pytestmark = pytest.mark.gpu
N_Q, N_KV, DIM, BLOCK, BLOCKS, WIDTH = 8, 2, 64, 16, 200, 40


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Run:
    """A cache and the state of four requests."""

    def __init__(self, seed):
        g = gen(seed)
        w = [1 + 0.3 * torch.randn(DIM, device=DEV, generator=g) for _ in range(2)]
        self.heads = dr.QKHeads(N_Q, N_KV, DIM, w[0].bfloat16(), w[1].bfloat16())
        self.cache = dr.KVCache.empty(BLOCKS, N_KV, BLOCK, DIM)
        for t in (self.cache.k, self.cache.v):
            t.view(torch.uint8).fill_(0x7F)
        self.lengths, self.table = ints([0] * 4), torch.full((4, WIDTH), -1, dtype=torch.int32, device=DEV)
        self.free, self.state = torch.randperm(BLOCKS, device=DEV, generator=g).int(), ints([BLOCKS, 0])

    def step(self, x, added, out=None, q=None, window=0, sinks=0):
        offsets, positions, runs = self.cache.extend(added, self.lengths, self.table, self.free, self.state, x.shape[0])
        q = self.heads.append(x, positions, runs, self.cache, out=q)
        return self.cache.attend(q, self.lengths, self.table, offsets, window=window, sinks=sinks, out=out), q, offsets


def rows(g, n):
    return torch.randn(n, (N_Q + 2 * N_KV) * DIM, device=DEV, generator=g).bfloat16()


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_prompts_and_tokens(window, sinks):
    run, g = Run(1), gen(2)
    for added in ([70, 1, 33, 0], [1, 1, 1, 20], [1, 5, 1, 1], [300, 1, -1, 1], [1, 1, 17, 1], [1, 1, 1, 1]):
        x = rows(g, sum(max(a, 0) for a in added) + 2)  # two rows that nobody owns
        out = torch.full((x.shape[0], N_Q * DIM), 7.0, dtype=torch.bfloat16, device=DEV)
        got, q, offsets = run.step(x, ints(added), out=out, q=torch.zeros_like(out), window=window, sinks=sinks)
        c = run.cache
        want, tol = attention(q, c.k, c.v, c.k_scale, c.v_scale, run.lengths.tolist(), offsets.tolist(), run.table, N_Q, window, sinks)
        mine = torch.arange(x.shape[0], device=DEV) < int(offsets[-1])
        assert ((got.double() - want).abs() <= tol)[mine].all() and (got[~mine] == 7).all() and (q[~mine] == 0).all()
        assert int(run.state[1]) == 0


def test_a_prompt_at_once_and_token_by_token():
    """The same tokens in one call, in chunks and one by one: the cache holds the same values (but below 2^-6 of a scale), so what a row
    sees differs by that, and by roundings."""
    n, outs = 150, []
    x = rows(gen(3), n)
    for chunks in ([150], [64, 1, 85], [1] * 150):
        run, at, got = Run(4), 0, []
        for c in chunks:
            got.append(run.step(x[at:at + c], ints([c, 0, 0, 0]))[0])
            at += c
        outs.append(torch.cat(got))
        assert run.lengths.tolist() == [150, 0, 0, 0] and int(run.state[0]) == BLOCKS - -(-150 // BLOCK)
    for o in outs[1:]:
        # a code below 2^-6 of its scale is off by at most 2^-10 of it twice, of values of some units: 2^-7 for a result covers it, and two
        # roundings to bf16
        assert (o.float() - outs[0].float()).abs().max() <= 2.0 ** -6 * outs[0].float().abs().max()


def test_captured_decode_steps():
    a, b, g = Run(5), Run(5), gen(6)
    prompt, added = rows(g, 100), ints([40, 25, 20, 15])
    for r in (a, b):
        r.step(prompt, added)
    one, x = ints([1] * 4), rows(g, 4)
    held = x.clone()
    b_state = [t.clone() for t in (b.lengths, b.table, b.free, b.state, b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale)]
    b.step(held, one)  # the module is loaded; the state is put back
    for t, s in zip((b.lengths, b.table, b.free, b.state, b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale), b_state):
        t.copy_(s)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros(4, N_Q * DIM, dtype=torch.bfloat16, device=DEV)
    with torch.cuda.graph(graph):
        b.step(held, one, out=out)
    for i in range(40):
        x = rows(g, 4)
        want = a.step(x, one)[0]
        held.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        assert torch.equal(a.lengths, b.lengths) and torch.equal(a.table, b.table) and torch.equal(a.state, b.state)


def test_two_graphs_with_their_own_caches_at_once():
    """Replayed on two streams together: no workspace is shared."""
    runs, graphs, outs, want = [Run(7), Run(8)], [], [], []
    added, x = ints([90, 70, 50, 30]), rows(gen(9), 240)
    for r in runs:
        r.step(x, added)
        q = torch.randn(4, N_Q * DIM, device=DEV, generator=gen(10)).bfloat16()
        want.append(r.cache.attend(q, r.lengths, r.table))
        out, graph = torch.zeros_like(q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(20):
                r.cache.attend(q, r.lengths, r.table, out=out)
        graphs.append(graph)
        outs.append((out, q))
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], w) for o, w in zip(outs, want))


@pytest.mark.parametrize("spec", [MID[0]["spec"], MID[2]["spec"]], ids=["dense", "moe"])
@pytest.mark.parametrize("tp", [1, 2])
def test_over_an_arena(spec, tp):
    """A layer's qkv product, norms, cache, attention and o product, the weights as dr_reshard has written them."""
    plan = dr.Plan(spec, tp=tp, tp_rank=tp - 1)
    flat = torch.randn(plan.info.flat_elems, device=DEV, generator=gen(11)) * 0.05
    arena = torch.empty(plan.info.dst_bytes, dtype=torch.uint8, device=DEV)
    plan.reshard(flat, arena)
    heads = plan.qk_heads(arena, "layers.0")
    assert heads.n_q_heads * tp == spec["n_q_heads"] and heads.n_kv_heads * tp == spec["n_kv_heads"] and heads.head_dim == spec["head_dim"]
    assert torch.equal(heads.q_norm, plan.view(arena, "layers.0.q_norm")[0].view(-1))
    x = torch.randn(5, spec["hidden"], device=DEV, generator=gen(12)).bfloat16()
    qkv = plan.linear(arena, "layers.0.qkv")(x)
    cache = dr.KVCache.empty(8, heads.n_kv_heads, 32, heads.head_dim)
    lengths, table, free, state = ints([0]), torch.full((1, 4), -1, dtype=torch.int32, device=DEV), ints(list(range(8))), ints([8, 0])
    offsets, positions, runs = cache.extend(ints([5]), lengths, table, free, state, 5)
    q = heads.append(qkv, positions, runs, cache)
    y = cache.attend(q, lengths, table, offsets)
    want, tol = attention(q, cache.k, cache.v, cache.k_scale, cache.v_scale, [5], [0, 5], table, heads.n_q_heads)
    assert ((y.double() - want).abs() <= tol).all()
    assert plan.linear(arena, "layers.0.o")(y).shape == (5, spec["hidden"])
    with pytest.raises(KeyError):
        plan.qk_heads(arena, "layers.99")


def test_the_example_runs():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rollout_attention.py")
    p = subprocess.run([sys.executable, path], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "tokens" in p.stdout, p.stdout[-2000:] + p.stderr[-2000:]
