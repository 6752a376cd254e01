"""The experts' operators together (``ExpertLayer``), on pooled lookups, against 64 bits.

The layer holds its weights, its inputs and its hidden values in 8 bits: the
reference takes the first two as held and the hidden values exact.  A hidden value
h is then off by half a step of e4m3, |h| 2^-4 + s 2^-10 with s its block's scale
(at most the block's largest |h| / 448), and by the products' rounding, far below;
an expert's output by the sum of |w| times that, and bf16's 2^-8; the joined row
by the weighted sum.
"""
import importlib.util
import os

import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def held(q, s, rows_each):
    """8-bit values and their scales as 64-bit numbers."""
    s = s.double().repeat_interleave(rows_each, -2)[..., :q.shape[-2], :].repeat_interleave(128, -1)[..., :q.shape[-1]]
    return q.double() * s


def reference(layer, x, scores, lo=0):
    r = ex.route(scores, layer.top, layer.mode, layer.bias, layer.groups, layer.top_groups, layer.scale)
    q, s = ex.quantize_fp8(x)
    X = held(q, s, 1)
    gate = layer.act == ex.EB_ACT_SILU_GATE
    half = layer.w_up.shape[1] // (2 if gate else 1)
    E = layer.E
    up = held(layer.w_up.reshape(-1, half, layer.K), layer.up_scales.reshape(-1, -(-half // 128), layer.up_scales.shape[2]), 128)
    up = up.reshape(E, -1, layer.K)
    down = held(layer.w_down, layer.down_scales, 128)
    out = torch.zeros(x.shape[0], layer.D, dtype=torch.float64, device=x.device)
    off = torch.zeros_like(out)
    for e in range(E):
        n, k = (r.ids == e + lo).nonzero(as_tuple=True)
        if not n.numel():
            continue
        v = X[n] @ up[e].t()
        h = v[:, :half] * torch.sigmoid(v[:, :half]) * v[:, half:] if gate else v.clamp(min=0)
        pad = torch.nn.functional.pad(h.abs(), (0, -half % 128))
        most = pad.view(n.numel(), -1, 128).amax(2).repeat_interleave(128, 1)[:, :half]
        dh = h.abs() * 2.0 ** -4 + most / 448 * 2.0 ** -10 + most * 2.0 ** -12
        y, dy = h @ down[e].t(), dh @ down[e].abs().t()
        w = r.weights[n, k].double()[:, None]
        out.index_add_(0, n, w * y)
        off.index_add_(0, n, w * (dy + (y.abs() + dy) * 2.0 ** -8) * (1 + 2.0 ** -10))
    return out, off


def layer_of(E, K, hidden, D, top, act, device, all_experts=None, lo=0, **kw):
    g = torch.Generator(device=device).manual_seed(E + K)
    N = 2 * hidden if act == ex.EB_ACT_SILU_GATE else hidden
    w_up = torch.randn(E, N, K, generator=g, device=device) * K ** -0.5
    w_down = torch.randn(E, D, hidden, generator=g, device=device) * hidden ** -0.5
    router = torch.randn(all_experts or E, K, generator=g, device=device) * K ** -0.5
    return ex.ExpertLayer(w_up, w_down, router, top, act=act, shard_lo=lo, **kw)


@pytest.mark.parametrize("B", [1, 3, 40, 700, 3000])
@pytest.mark.parametrize("E,K,hidden,D,top,act", [(8, 256, 128, 64, 2, ex.EB_ACT_SILU_GATE), (5, 378, 200, 100, 3, ex.EB_ACT_RELU),
                                                  (16, 512, 300, 256, 4, ex.EB_ACT_SILU_GATE)])
def test_layer(B, E, K, hidden, D, top, act, device):
    layer = layer_of(E, K, hidden, D, top, act, device)
    x = torch.randn(B, K, generator=torch.Generator(device=device).manual_seed(B), device=device) * 0.3
    scores = torch.randn(B, E, generator=torch.Generator(device=device).manual_seed(B + 1), device=device)
    scores[B // 2] = -float("inf")  # a token without experts
    got = layer.forward(x, scores)
    want, off = reference(layer, x, scores)
    assert ((got.double() - want).abs() <= off).all()
    assert (got[B // 2] == 0).all()


def test_shards_add_up(device):
    """Each of four GPUs' shares gives a partial result; their sum is the whole."""
    E, K, hidden, D, top, B = 12, 256, 128, 128, 3, 200
    whole = layer_of(E, K, hidden, D, top, ex.EB_ACT_SILU_GATE, device)
    x = torch.randn(B, K, generator=torch.Generator(device=device).manual_seed(2), device=device)
    scores = torch.randn(B, E, generator=torch.Generator(device=device).manual_seed(3), device=device)
    parts = []
    for lo in range(0, E, 3):
        part = layer_of(E, K, hidden, D, top, ex.EB_ACT_SILU_GATE, device)
        part.E, part.shard_lo = 3, lo
        for name in ("w_up", "up_scales", "w_down", "down_scales"):
            setattr(part, name, getattr(part, name)[lo:lo + 3])
        parts.append(part.forward(x, scores))
    total = eb.sum_partials(torch.stack(parts), B, 1, D)
    want, off = reference(whole, x, scores)
    assert ((total.double() - want).abs() <= off).all()
    assert ((whole.forward(x, scores).double() - want).abs() <= off).all()


def test_example_runs(device):
    spec = importlib.util.spec_from_file_location("pooled_experts", os.path.join(ROOT, "examples", "pooled_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    et, layer = m.build(tables=3, rows=5000, dim=64, experts=8, hidden=128, out=96, top=2)
    ids, offsets = m.batch(et, 33, 7)
    pooled, out = m.step(et, layer, ids, offsets, 33)
    want, off = reference(layer, pooled, pooled @ layer.router.t())
    assert out.shape == (33, 96) and ((out.double() - want).abs() <= off).all()
    et.close()


def test_refusals(device):
    w_up, w_down, router = (torch.zeros(2, 6, 8, device=device), torch.zeros(2, 4, 3, device=device), torch.zeros(2, 8, device=device))
    ex.ExpertLayer(w_up, w_down, router, 1)
    for bad in ((w_up[:, :5], w_down, router), (w_up, w_down[:1], router), (w_up, w_down, router[:, :7]), (w_up[0], w_down, router)):
        with pytest.raises(ValueError):
            ex.ExpertLayer(*bad, 1)


def test_one_layer_on_two_streams(device):
    """A stream that has not waited for another's call does not need that call's results."""
    layer = layer_of(8, 256, 128, 64, 2, ex.EB_ACT_RELU, device)
    x = torch.randn(50, 256, device=device)
    scores = torch.randn(50, 8, device=device)
    want = layer_of(8, 256, 128, 64, 2, ex.EB_ACT_RELU, device).forward(x, scores)
    torch.cuda.synchronize()
    late, early = torch.cuda.Stream(), torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=device)
    torch.cuda.synchronize()
    with torch.cuda.stream(late):
        for _ in range(20):  # holds this stream's call back
            big = big @ big * 1e-3
        first = layer.forward(x, scores)
    with torch.cuda.stream(early):
        second = layer.forward(x, scores)
    torch.cuda.synchronize()
    assert torch.equal(first, want) and torch.equal(second, want)
