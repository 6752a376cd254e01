"""``ExpertTraining`` with ``exact_router``: the router's gradient from what it read and its outputs' gradients, both in fp32.

A sum over B tokens in fp32, in any order: (B + 2) u of the sum of the sizes, u = 2^-24."""
import pytest
import torch

from paper_2512_05831_amd import train
from train_util import U, generator
from test_gpu_expert_training import layer_of

pytestmark = pytest.mark.gpu


def read_by(layer, x):
    """What the router reads: x, or the layer norm's output in x's type."""
    if layer.norm_weight is None:
        return x
    return train.layer_norm(x, layer.norm_weight, layer.norm_bias, layer.eps, out_dtype=x.dtype).y


@pytest.mark.parametrize("B", [0, 1, 7, 300, 2000])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_of_what_it_read(B, norm, dtype, device):
    layer, plain = (layer_of(8, 200, 64, 32, 2, device, norm=norm, **kw) for kw in (dict(exact_router=True), {}))
    g = generator(device, B)
    x, dout = torch.randn(B, 200, generator=g, device=device).to(dtype), torch.randn(B, 32, generator=g, device=device)
    out, s = layer.forward(x)
    grads, mid = layer._backward(s, dout)
    ds, read = mid["dscores"].double(), read_by(layer, x).double()
    assert torch.equal(s.read.double(), read) and grads.router.dtype == torch.float32
    assert ((grads.router.double() - ds.t() @ read).abs() <= (B + 2) * U * (ds.abs().t() @ read.abs())).all()
    # All else is as without it, and nothing more is kept there.
    want, saved = plain.forward(x)
    other = plain.backward(saved, dout)
    assert saved.read is None and torch.equal(out, want)
    for name in ("x", "w_up", "w_down", "norm_weight", "norm_bias"):
        a, b = getattr(grads, name), getattr(other, name)
        assert (a is None and b is None) or torch.equal(a, b)


def test_graph(device):
    layer = layer_of(8, 256, 128, 64, 2, device, exact_router=True)
    x, dout = torch.randn(1000, 256, generator=generator(device, 2), device=device), torch.randn(1000, 64, generator=generator(device, 3), device=device)

    def step():
        out, s = layer.forward(x)
        return (out, *layer.backward(s, dout))
    side = torch.cuda.Stream(device)
    side.wait_stream(torch.cuda.current_stream(device))
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for replay in range(4):
        x.copy_(torch.randn(1000, 256, generator=generator(device, 10 + replay), device=device))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b), replay
