"""``ExpertTraining`` where torch casts products by itself: the router's stay in fp32, and the results the same bits."""
import pytest
import torch

from train_util import generator
from test_gpu_expert_training import layer_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_under_autocast(dtype, exact, norm, device):
    layer = layer_of(8, 256, 128, 64, 2, device, norm=norm, exact_router=exact)
    x, dout = torch.randn(50, 256, generator=generator(device, 2), device=device), torch.randn(50, 64, generator=generator(device, 3), device=device)
    want, s = layer.forward(x)
    want_grads = layer.backward(s, dout)
    with torch.autocast("cuda", dtype=dtype):
        out, saved = layer.forward(x)
        grads = layer.backward(saved, dout)
    outside = layer.backward(saved, dout)
    assert saved.scores.dtype == torch.float32 and torch.equal(out, want)
    for a, b, c in zip(want_grads, grads, outside):
        assert (a is None and b is None and c is None) or (torch.equal(a, b) and torch.equal(a, c) and a.dtype == b.dtype)
