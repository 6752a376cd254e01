"""The gate of eb_activation and eb_activation_backward over all of fp32's range.

The quotient g / (1 + exp(-g)) is within 4 + |g| ulp of fp32, or 2^-119, whatever g: the
bound does not grow past |g| = 88, from where p = 1 / (1 + exp(-g)) is 1, or below 2^-126
and may be 0.  In the gradients such a p costs at most 2^-126 of the other factors, which
are dh (or 1, where dh p leaves fp32's normal numbers), u and 1 + |g|, with |g| up to 104:
past that p is below 2^-149.  Infinities give what the formula gives.
"""
import pytest
import torch

from paper_2512_05831_amd import experts as ex, train
from train_util import FP8, U, check, check8

pytestmark = pytest.mark.gpu
LOW = [-80.0, -86.0, -87.0, -87.25, -87.5, -88.0, -88.5, -88.72, -88.73, -89.0, -95.0, -100.0, -103.0, -104.0, -150.0, -200.0, -1e3, -1e4, -1e6,
       -3e7, -1e10, -1e20, -1e30, -1e37, -1e38, -3e38]
HIGH = [80.0, 87.0, 88.0, 88.73, 90.0, 104.0, 150.0, 1e4, 1e10, 1e30, 1e38, 3e38, 0.0, -0.0, 1.0, -1.0]


def forward(v):
    g, u = v.chunk(2, 1)
    q = g * torch.sigmoid(g)
    eq = torch.maximum(q.abs() * (4 + g.abs().clamp(max=88)) * 2 * U, torch.full_like(q, 2.0 ** -119))
    return q * u, (eq + U * q.abs()) * u.abs()


def backward(dh, v):
    g, u = v.chunk(2, 1)
    p, q, far = torch.sigmoid(g), torch.sigmoid(-g), g.abs().clamp(max=88)
    T, ep = 1 + g * q, (5 + far) * 2 * U
    eT = far * (ep * p + 2 * U) + 2 * U * (1 + (g * q).abs())
    lost = 2.0 ** -125 * dh.abs().clamp(min=1) * g.abs().clamp(max=104).add(1)
    dg, du = dh * u * p * T, dh * g * p
    edg = (dh * u).abs() * p * (T.abs() * (ep + 8 * U) + eT) + lost * u.abs()
    return torch.cat([dg, du], 1), torch.cat([edg, (ep + 6 * U) * du.abs() + lost], 1)


def check_both(v, s, values, dh, out):
    h, dv = train.activation(v, s, out_dtype=out), train.activation_backward(dh, v, s, out_dtype=out)
    if out == FP8:
        check8(*h, *forward(values))
        check8(*dv, *backward(dh.double(), values))
    else:
        check(h, *forward(values), out)
        check(dv, *backward(dh.double(), values), out)


@pytest.mark.parametrize("v_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1.0, 1e-3, -1e3])
def test_floating(v_type, size, device):
    """u small enough that products with a g of 1e38 stay finite."""
    for g in (LOW, HIGH, LOW + HIGH):
        g = torch.tensor(g, device=device)
        for u in (0.75, -1e-4):
            v = torch.cat([g, torch.full_like(g, u)])[None].to(v_type).contiguous()
            check_both(v, None, v.double(), torch.full((1, g.numel()), size * 1e-3, device=device), torch.float32)


@pytest.mark.parametrize("cols", [128, 256, 136, 100, 21])
@pytest.mark.parametrize("top", [100.0, 300.0, 1e4, 1e30, 3e38])
def test_eight_bits(cols, top, device):
    """Every kernel of 8-bit values: whole blocks, blocks across the border, rows that end inside a chunk."""
    g = -top * torch.linspace(0.01, 1, cols, device=device).repeat(5, 1)
    u = torch.linspace(-1, 1, cols, device=device).repeat(5, 1) * torch.tensor([1.0, 1e-3, 1e3, 1e10, -1.0], device=device)[:, None]
    parts = [ex.quantize_fp8(x) for x in (g, u)]
    whole = torch.cat([g, u], 1)
    q, s = ex.quantize_fp8(whole)
    if cols % 128 == 0:  # each half in its own blocks
        q, s = q.clone(), torch.cat([p[1] for p in parts], 1)
        q.view(torch.uint8)[:, :cols], q.view(torch.uint8)[:, cols:] = (p[0].view(torch.uint8) for p in parts)
    values = q.double() * s.double().repeat_interleave(128, 1)[:, :2 * cols]
    dh = torch.linspace(1, -2, cols, device=device).repeat(5, 1) * 1e-2
    for out in (FP8, torch.float32):
        for dh_type in (torch.float32, torch.bfloat16):
            check_both(q, s, values, dh.to(dh_type), out)


def test_infinities(device):
    """-infinity: p = 0, and 0 times infinity is NaN; infinity: p = 1, but 1 + g (1 - p) is NaN."""
    v = torch.tensor([[-float("inf"), float("inf"), float("nan"), -1e38, 2.0] + [0.5] * 5], device=device)
    dh = torch.ones(1, 5, device=device)
    h, dv = train.activation(v, out_dtype=torch.float32)[0], train.activation_backward(dh, v, out_dtype=torch.float32)[0]
    assert h.isnan().tolist() == [True, False, True, False, False] and h[1] == float("inf") and h[3] == 0
    assert dv[:5].isnan().tolist() == [True, True, True, False, False] and dv[5:].isnan().tolist() == [True, False, True, False, False]
    assert dv[6] == float("inf") and dv[3] == 0 and dv[8] == 0
