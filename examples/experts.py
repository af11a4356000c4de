"""The experts of one MoE layer across a role switch: fp8 rollout, then a training step, from one flat fp32 master.

    python examples/experts.py

Rollout: dr_reshard writes the layer's experts as e4m3 with block scales; tokens are routed, gathered and quantised
(quant_rows with row_index), multiplied by expert (w13), put through SwiGLU and quantised again in one pass, multiplied by w2 and
combined.  Training: a bf16 plan gives the same layer for compute; dgrad and wgrad run back through both products, the fp32
gradients land in the arena of a DR_F32 plan, and dr_reshard_inverse takes them to the positions of the flat master, where
an SGD step is one axpy.  The printed loss falls.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch
import torch.nn.functional as F

import paper_2607_22614_b200 as dr

SPEC = dict(n_layers=1, hidden=512, n_q_heads=8, n_kv_heads=4, head_dim=64, ffn=0, vocab=1024, n_experts=8, moe_ffn=192, tied=0,
            qk_norm=1)
TOP = 2


def route(x, router):
    """(token of each row sorted by expert, its weight, offsets): every token goes to its TOP best experts."""
    weight, expert = (x.float() @ router.float().t()).softmax(-1).topk(TOP, dim=-1)
    order = expert.reshape(-1).argsort(stable=True)
    offsets = torch.zeros(SPEC["n_experts"] + 1, dtype=torch.int32, device=x.device)
    offsets[1:] = torch.bincount(expert.reshape(-1), minlength=SPEC["n_experts"]).cumsum(0)
    return order // TOP, weight.reshape(-1)[order], offsets


def combine(rows, token, weight, tokens):
    out = torch.zeros(tokens, rows.shape[1], device=rows.device)
    return out.index_add_(0, token, rows.float() * weight[:, None])


def rollout(master, x):
    plan = dr.Plan(SPEC, dtype=dr.DR_FP8_E4M3_B128)
    arena = torch.empty(plan.info.dst_bytes, dtype=torch.uint8, device=x.device)
    plan.reshard(master, arena)
    w13, w2 = plan.linear(arena, "layers.0.w13"), plan.linear(arena, "layers.0.w2")
    token, weight, offsets = route(x, plan.view(arena, "layers.0.router")[0])
    h = w13.forward(*dr.quant_rows(x, row_index=token), offsets)
    y = w2.forward(*dr.quant_rows(h, swiglu=True), offsets)
    return combine(y, token, weight, x.shape[0])


def train_step(master, x, target, rate):
    """One SGD step on the experts for mean((y - target)^2); the new master and the loss before the step."""
    plan, grads = dr.Plan(SPEC), dr.Plan(SPEC, dtype=dr.DR_F32)
    arena = torch.empty(plan.info.dst_bytes, dtype=torch.uint8, device=x.device)
    plan.reshard(master, arena)
    w13, w2 = plan.linear(arena, "layers.0.w13"), plan.linear(arena, "layers.0.w2")
    token, weight, offsets = route(x, plan.view(arena, "layers.0.router")[0])
    rows = x[token]
    h = w13.forward(rows, None, offsets)
    gate, up = h.float().chunk(2, dim=-1)
    act = (F.silu(gate) * up).bfloat16()
    y = w2.forward(act, None, offsets)
    diff = combine(y, token, weight, x.shape[0]) - target
    # back through the combination, w2, SwiGLU and w13
    dy = (diff[token] * weight[:, None] * (2.0 / diff.numel())).bfloat16()
    dact = w2.dgrad(dy, offsets, out_dtype=torch.float32)
    s = torch.sigmoid(gate)
    dh = torch.cat([dact * up * s * (1 + gate * (1 - s)), dact * F.silu(gate)], dim=-1).bfloat16()
    garena = torch.zeros(grads.info.dst_bytes, dtype=torch.uint8, device=x.device)
    w2.wgrad(act, dy, offsets, out=grads.view(garena, "layers.0.w2")[0])
    w13.wgrad(rows, dh, offsets, out=grads.view(garena, "layers.0.w13")[0])
    flat = torch.zeros_like(master)
    grads.reshard_inverse(garena, flat)
    return master - rate * flat, float(diff.square().mean())


def main(steps=5):
    torch.manual_seed(0)
    dev = torch.device("cuda:0")
    elems = dr.Plan(SPEC, host_only=True).info.flat_elems
    master = torch.randn(elems, device=dev) * 0.05
    x = torch.randn(333, SPEC["hidden"], device=dev).bfloat16()
    target = torch.randn(333, SPEC["hidden"], device=dev) * 0.5
    losses = []
    for _ in range(steps):
        master, loss = train_step(master, x, target, rate=100.0)
        losses.append(loss)
    fp8 = float((rollout(master, x) - target).square().mean())
    print("loss by step:", " ".join(f"{v:.4f}" for v in losses), "| after the switch to fp8 rollout:", f"{fp8:.4f}")
    return losses, fp8


if __name__ == "__main__":
    main()
