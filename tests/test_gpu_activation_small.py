"""eb_activation_backward between 8-bit matrices where dh u lies below what a factor of 448 / largest can be made of (448 x 2^-126)
before u has its scale, and above it with that."""
import pytest
import torch

from paper_2512_05831_amd import train
from train_util import FP8, check8, generator
from test_gpu_activation import GATE, backward

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -149


@pytest.mark.parametrize("dh_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [128, 384, 100])
def test_gate_of_small_gradients(cols, dh_type, device):
    """dh u below the floor before the scale of u, above it with that."""
    g = generator(device, cols)
    rows = 6
    q = torch.randn(rows, 2 * cols + 15 & -16, generator=g, device=device).clamp(-4, 4).to(FP8)[:, :2 * cols]
    s = torch.ones((2 * cols + 127) // 128, rows, device=device).t()
    s[:, -(-cols // 128):] = torch.tensor([1.0, 2.0 ** 8, 2.0 ** 20, 2.0 ** 60, 2.0 ** 100, 2.0 ** -5], device=device)[:, None]
    dh = ((1 + torch.rand(rows, cols, generator=g, device=device)) * 6e-38).to(dh_type)
    values = q.double() * s.double().repeat_interleave(128, 1)[:, :2 * cols]
    p = torch.sigmoid(values[:, :cols])
    # dh p as long as it is normal; products with u rounded to multiples of 2^-149.
    assert float((dh.double() * p).min()) > 2.0 ** -130
    want, err = backward(dh.double(), values, GATE)
    gg, u = values.chunk(2, 1)
    tiny = 4 * LEAST * torch.cat([(1 + u.abs()) * (1 + gg.abs()), 1 + gg.abs()], 1)
    gone = torch.where(dh.double() * p < 2.0 ** -126, dh.double() * p, 0.0)
    tiny += torch.cat([gone * u.abs() * (1 + gg.abs()), gone * gg.abs()], 1)
    err = err - 2.0 ** -116 * torch.cat([(dh.double() * u).abs() * (1 + gg.abs()), (dh.double() * gg).abs()], 1)  # that bound's slack for a p of 0
    check8(*train.activation_backward(dh, q, s, out_dtype=FP8), want, err.clamp(min=0) + tiny)
