"""The attention of one layer in the rollout role, from an arena's weights: prompts in one step, then tokens one by one from a graph.

    python examples/rollout_attention.py

dr_reshard writes the layer's weights; a step is KVCache.extend (block tables, positions and the runs of slots from the lengths on the
GPU), the qkv product, QKHeads.append (norms and rotation, keys and values into the 8-bit cache), KVCache.attend and the o product.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2607_22614_b200 as dr

SPEC = dict(n_layers=1, hidden=512, n_q_heads=8, n_kv_heads=4, head_dim=64, ffn=1024, vocab=1024, tied=0, qk_norm=1)
BLOCKS, BLOCK_TOKENS, WIDTH = 256, 16, 32


class Layer:
    def __init__(self, master, requests):
        dev = master.device
        self.plan = dr.Plan(SPEC)
        self.arena = torch.empty(self.plan.info.dst_bytes, dtype=torch.uint8, device=dev)
        self.plan.reshard(master, self.arena)
        self.qkv, self.o = self.plan.linear(self.arena, "layers.0.qkv"), self.plan.linear(self.arena, "layers.0.o")
        self.heads = self.plan.qk_heads(self.arena, "layers.0")
        self.cache = dr.KVCache.empty(BLOCKS, SPEC["n_kv_heads"], BLOCK_TOKENS, SPEC["head_dim"])
        self.lengths = torch.zeros(requests, dtype=torch.int32, device=dev)
        self.table = torch.full((requests, WIDTH), -1, dtype=torch.int32, device=dev)
        self.free = torch.arange(BLOCKS, dtype=torch.int32, device=dev)
        self.state = torch.tensor([BLOCKS, 0], dtype=torch.int32, device=dev)

    def step(self, x, added):
        """x: the hidden states of all requests' new tokens, one request behind another; added: how many each request has."""
        offsets, positions, runs = self.cache.extend(added, self.lengths, self.table, self.free, self.state, x.shape[0])
        q = self.heads.append(self.qkv(x), positions, runs, self.cache)
        return self.o(self.cache.attend(q, self.lengths, self.table, offsets))


def main(steps=20):
    torch.manual_seed(0)
    dev = torch.device("cuda:0")
    master = torch.randn(dr.Plan(SPEC, host_only=True).info.flat_elems, device=dev) * 0.05
    prompts = [37, 5, 120, 64]
    layer = Layer(master, len(prompts))
    x = torch.randn(sum(prompts), SPEC["hidden"], device=dev).bfloat16()
    y = layer.step(x, torch.tensor(prompts, dtype=torch.int32, device=dev))
    one = torch.ones(len(prompts), dtype=torch.int32, device=dev)
    token = torch.randn(len(prompts), SPEC["hidden"], device=dev).bfloat16()
    layer.step(token, one)  # (an ordinary step loads what the graph needs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.step(token, one)
    for _ in range(steps):
        graph.replay()
        token.copy_(out)  # stands for the rest of the model
    torch.cuda.synchronize()
    print("tokens held:", layer.lengths.tolist(), "| blocks left:", int(layer.state[0]), "| finite:", bool(torch.isfinite(out).all() and torch.isfinite(y).all()))
    return layer.lengths.tolist()


if __name__ == "__main__":
    main()
