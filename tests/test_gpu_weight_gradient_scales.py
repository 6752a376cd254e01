"""What eb_weight_gradient keeps of slots whose scales are small beside others'.

Products are within 2^-20 of exact, and where neither operand is bfloat16 and one has scales
within 2^-34 of the largest that the scales of the expert's slots allow: of each product, not
of a sum's, so that a column whose only value lies in one slot shows it.  A product in fp32
is rounded twice (2^-23), and nothing but zeros is added to it.
"""
import pytest
import torch

from paper_2512_05831_amd import train
from train_util import FP8, U, check, generator
from test_gpu_weight_gradient import BF16, F32, HALF

pytestmark = pytest.mark.gpu


def column_major(s):
    return s.t().contiguous().t()


@pytest.mark.parametrize("power", [0, 4, 10, 13, 16, 20, 25, 30, 40])
@pytest.mark.parametrize("other,own_x", [(FP8, False), (HALF, False), (HALF, True)])
@pytest.mark.parametrize("large_at", [0, 77, 199])
def test_one_value_in_a_column(power, other, own_x, large_at, device):
    """A slot of large scale, zero in all columns but the first, among slots of scale 2^-power; every other column has
    its value in one of those."""
    g = generator(device, power)
    M, N, K = 200, 300, 130
    # Values of e4m3 with all their bits, the largest and the smallest among them.
    codes = torch.arange(1, 127, dtype=torch.uint8, device=device).view(FP8)
    pick = lambda r, c: codes.view(torch.uint8)[torch.randint(0, 126, (r, c), generator=g, device=device)]  # noqa: E731
    q = torch.zeros(M, N + 15 & -16, dtype=torch.uint8, device=device)
    slot = torch.randint(0, M - 1, (N,), generator=g, device=device)
    slot = torch.where(slot >= large_at, slot + 1, slot)
    q[slot, torch.arange(N, device=device)] = pick(1, N)[0]
    q[:, 0] = 0
    q[large_at, 0] = codes.view(torch.uint8)[-1]
    q = q.view(FP8)[:, :N]
    s = (1 + torch.rand(M, 3, generator=g, device=device)) * 2.0 ** -power
    s[large_at] = 1.75
    s = column_major(s)
    if other == FP8:
        x = pick(M, K + 15 & -16).view(FP8)[:, :K]
        xs = column_major(1 + torch.rand(M, 2, generator=g, device=device))
        xv = x.double() * xs.double().repeat_interleave(128, 1)[:, :K]
        most = 448.0 ** 2 * float(s.max()) * float(xs.max())
    else:
        x = torch.randn(M, K, generator=g, device=device).to(HALF)
        xs, xv = None, x.double()
        most = 448.0 * float(s.max()) * float(xv.abs().max())
    dv = q.double() * s.double().repeat_interleave(128, 1)[:, :N]
    want = dv.t() @ xv
    for out in (F32, HALF, BF16):
        if out == HALF and float(want.abs().max()) > 6e4:
            continue
        if own_x:
            got, of = train.weight_gradient(x, q, x_scales=s, out_dtype=out), want.t()
        else:
            got, of = train.weight_gradient(q, x, dy_scales=s, x_scales=xs, out_dtype=out), want
        check(got, of, (2.0 ** -20 + 2 * U) * of.abs() + 2.0 ** -34 * most, out)
