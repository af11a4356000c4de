"""The experts example, end to end, against the same layer in plain 64-bit torch with autograd."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

import paper_2607_22614_b200 as dr

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("experts_example", os.path.join(ROOT, "examples", "experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain(ex, w13, w2, x, token, weight, offsets):
    ends, out = offsets.tolist(), torch.zeros(x.shape[0], w2.shape[1], dtype=torch.float64, device=x.device)
    for e in range(ex.SPEC["n_experts"]):
        t = token[ends[e]:ends[e + 1]]
        gate, up = (x[t] @ w13[e].t()).chunk(2, -1)
        out = out.index_add(0, t, (F.silu(gate) * up) @ w2[e].t() * weight[ends[e]:ends[e + 1], None])
    return out


def _layer(ex, plan, arena):
    e, h, f = ex.SPEC["n_experts"], ex.SPEC["hidden"], ex.SPEC["moe_ffn"]
    return (plan.view(arena, "layers.0.w13")[0].double().view(e, 2 * f, h), plan.view(arena, "layers.0.w2")[0].double().view(e, h, f))


def test_a_training_step_moves_the_master_along_the_gradient():
    ex = _example()
    dev = torch.device("cuda:0")
    torch.manual_seed(1)
    plan, wide = dr.Plan(ex.SPEC), dr.Plan(ex.SPEC, dtype=dr.DR_F32)
    master = torch.randn(plan.info.flat_elems, device=dev) * 0.05
    x, target = torch.randn(77, 512, device=dev).bfloat16(), torch.randn(77, 512, device=dev)
    arena = torch.empty(plan.info.dst_bytes, dtype=torch.uint8, device=dev)
    plan.reshard(master, arena)
    w13, w2 = (w.requires_grad_() for w in _layer(ex, plan, arena))
    token, weight, offsets = ex.route(x, plan.view(arena, "layers.0.router")[0])
    loss = (_plain(ex, w13, w2, x.double(), token, weight.double(), offsets) - target).square().mean()
    loss.backward()
    after, got = ex.train_step(master, x, target, rate=1.0)
    assert abs(got / loss.item() - 1) < 1e-2
    step = torch.empty(wide.info.dst_bytes, dtype=torch.uint8, device=dev)
    wide.reshard(master - after, step)
    # gradients come through bf16 activations and bf16 dy: each is off by some 2^-8 of its size, independently
    for name, grad in (("layers.0.w13", w13.grad), ("layers.0.w2", w2.grad)):
        got = wide.view(step, name)[0].double()
        want = grad.reshape(got.shape)
        assert (got - want).norm() < 2e-2 * want.norm(), name
    assert wide.view(step, "layers.0.qkv")[0].abs().max() == 0 and wide.view(step, "embed")[0].abs().max() == 0


def test_fp8_rollout_of_the_layer():
    ex = _example()
    dev = torch.device("cuda:0")
    torch.manual_seed(2)
    plan = dr.Plan(ex.SPEC)
    master = torch.randn(plan.info.flat_elems, device=dev) * 0.05
    x = torch.randn(77, 512, device=dev).bfloat16()
    arena = torch.empty(plan.info.dst_bytes, dtype=torch.uint8, device=dev)
    plan.reshard(master, arena)
    w13, w2 = _layer(ex, plan, arena)
    token, weight, offsets = ex.route(x, plan.view(arena, "layers.0.router")[0])
    want = _plain(ex, w13, w2, x.double(), token, weight.double(), offsets)
    got = ex.rollout(master, x).double()
    # e4m3 rounds to 2^-4 at worst, 2^-5.8 on average (rms); four roundings (x, w13, activation, w2) add in squares
    assert (got - want).norm() < 2 * 2.0 ** -5.8 * 2 * want.norm()


def test_the_example_learns():
    losses, fp8 = _example().main()
    assert all(b < a for a, b in zip(losses, losses[1:])) and fp8 < losses[0]
