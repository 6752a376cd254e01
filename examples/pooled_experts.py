"""A ranking model's first two stages on one MI355X: pooled lookups, then a mixture of experts.

``python examples/pooled_experts.py`` pools the rows that a batch's ids name
(8 tables of 1M x 128, sum pooling), sends the pooled vectors through a layer of
gated experts in 8 bits, and prints what each step takes.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2512_05831_amd import eb, experts as ex


def build(tables=8, rows=1_000_000, dim=128, experts=32, hidden=1024, out=512, top=4, seed=0):
    """Tables and an expert layer of random weights."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = tables * dim
    et = eb.EmbeddingBagTables([0.01 * torch.randn(rows, dim, generator=g, device="cuda") for _ in range(tables)])
    w_up = torch.randn(experts, 2 * hidden, width, generator=g, device="cuda") * width ** -0.5
    w_down = torch.randn(experts, out, hidden, generator=g, device="cuda") * hidden ** -0.5
    router = torch.randn(experts, width, generator=g, device="cuda") * width ** -0.5
    return et, ex.ExpertLayer(w_up, w_down, router, top)


def batch(et, bags, pooling, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = et.rows[0]
    ids = torch.randint(0, rows, (et.T * bags * pooling,), generator=g, device="cuda")
    return ids, torch.arange(0, et.T * bags * pooling + 1, pooling, device="cuda")


def step(et, layer, ids, offsets, bags):
    pooled = et.forward(ids, offsets, bags, mode=eb.EB_SUM | eb.EB_HINT_STREAM_ROWS)
    return pooled, layer.forward(pooled)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--bags", type=int, default=2048)
    p.add_argument("--pooling", type=int, default=40)
    p.add_argument("--steps", type=int, default=50)
    a = p.parse_args()
    et, layer = build()
    ids, offsets = batch(et, a.bags, a.pooling)
    step(et, layer, ids, offsets, a.bags)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    torch.cuda.synchronize()
    marks[0].record()
    for _ in range(a.steps):
        pooled = et.forward(ids, offsets, a.bags, mode=eb.EB_SUM | eb.EB_HINT_STREAM_ROWS)
    marks[1].record()
    for _ in range(a.steps):
        out = layer.forward(pooled)
    marks[2].record()
    torch.cuda.synchronize()
    print(f"{a.bags} bags: pooled lookups {marks[0].elapsed_time(marks[1]) / a.steps * 1e3:.1f} us, "
          f"{layer.top} of {layer.E} experts {marks[1].elapsed_time(marks[2]) / a.steps * 1e3:.1f} us; "
          f"out {tuple(out.shape)}, finite: {bool(torch.isfinite(out).all())}")


if __name__ == "__main__":
    main()
