"""Training a mixture of experts on pooled lookups on one MI355X.

``python examples/train_experts.py`` pools the rows that a batch's ids name (8 tables
of 1M x 128, sum pooling; the tables stay as they are), sends the pooled vectors through
a layer norm and a layer of gated experts, takes the squared error against a random
target, and follows the gradients of all the layer's weights, whose forward values waited
in 8 bits.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2512_05831_amd import eb, train


def build(tables=8, rows=1_000_000, dim=128, experts=32, hidden=1024, out=512, top=4, seed=0):
    """Tables and an expert layer of random weights."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = tables * dim
    et = eb.EmbeddingBagTables([0.01 * torch.randn(rows, dim, generator=g, device="cuda") for _ in range(tables)])
    w_up = torch.randn(experts, 2 * hidden, width, generator=g, device="cuda") * width ** -0.5
    w_down = torch.randn(experts, out, hidden, generator=g, device="cuda") * hidden ** -0.5
    router = torch.randn(experts, width, generator=g, device="cuda") * width ** -0.5
    return et, train.ExpertTraining(w_up, w_down, router, top, norm_weight=torch.ones(width, device="cuda"),
                                    norm_bias=torch.zeros(width, device="cuda"))


def batch(et, bags, pooling, out, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, et.rows[0], (et.T * bags * pooling,), generator=g, device="cuda")
    return ids, torch.arange(0, et.T * bags * pooling + 1, pooling, device="cuda"), torch.randn(bags, out, generator=g, device="cuda")


def step(et, layer, ids, offsets, target, bags, rate):
    """One step of plain gradient descent; the loss and the gradients."""
    pooled = et.forward(ids, offsets, bags, mode=eb.EB_SUM | eb.EB_HINT_STREAM_ROWS)
    out, saved = layer.forward(pooled)
    off = out - target
    grads = layer.backward(saved, off * (2 / off.numel()))
    for weight, grad in ((layer.w_up, grads.w_up), (layer.w_down, grads.w_down), (layer.router, grads.router),
                         (layer.norm_weight, grads.norm_weight), (layer.norm_bias, grads.norm_bias)):
        weight.sub_(grad, alpha=rate)
    layer.refresh()
    return off.square().mean(), grads


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--bags", type=int, default=2048)
    p.add_argument("--pooling", type=int, default=40)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--rate", type=float, default=100.0)
    a = p.parse_args()
    et, layer = build()
    ids, offsets, target = batch(et, a.bags, a.pooling, layer.D)
    first, _ = step(et, layer, ids, offsets, target, a.bags, a.rate)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        last, _ = step(et, layer, ids, offsets, target, a.bags, a.rate)
    end.record()
    torch.cuda.synchronize()
    print(f"{a.bags} bags, {layer.top} of {layer.E} experts: {begin.elapsed_time(end) / a.steps:.2f} ms a step; "
          f"squared error {float(first):.4f}, after {a.steps} steps more {float(last):.4f}")


if __name__ == "__main__":
    main()
