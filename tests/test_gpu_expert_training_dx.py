"""The type of x's gradient in ``ExpertTraining.backward``: the joined rows' fp32 sums go into the norm's gradients, and out, in
the type asked for.  Errors as in the tests of layer norm's gradients: the sums' own are (experts + top + 4) u of their
sizes (u = 2^-24), the norm passes them on."""
import pytest
import torch

from paper_2512_05831_amd import train
from train_util import FP8, HALF_STEP, LEAST, U, WIDE, check, generator, held
from test_gpu_expert_training import layer_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", [None] + WIDE)
def test_type(norm, dtype, device):
    B, E, top = 200, 8, 3
    layer = layer_of(E, 256, 128, 64, top, device, norm=norm)
    g = generator(device, 1)
    x, dout = torch.randn(B, 256, generator=g, device=device), torch.randn(B, 64, generator=g, device=device)
    _, s = layer.forward(x)
    grads, mid = layer._backward(s, dout, dtype)
    of = dtype or (torch.bfloat16 if norm else torch.float32)
    slots, router, ds = s.route.slots.long(), layer.router.double(), mid["dscores"].double()
    back = mid["dslots"].double()[slots]
    dx, size = back.sum(1) + ds @ router, back.abs().sum(1) + ds.abs() @ router.abs()
    err = (E + top + 4) * U * size
    if not norm:
        check(grads.x, dx, err, of)
    else:
        err = err + (dx.abs() + err) * HALF_STEP[of] + LEAST[of]  # into the norm's gradients
        n, rs, wt = held(*s.kept), s.rstd.double()[:, None], layer.norm_weight.double()
        gg, ge = dx * wt, err * wt.abs()
        want = rs * (gg - gg.mean(1, keepdim=True) - n * (gg * n).mean(1, keepdim=True))
        slack = rs * (ge + ge.mean(1, keepdim=True) + n.abs() * (ge * n.abs()).mean(1, keepdim=True))
        slack = slack + 64 * U * rs * (gg.abs() + gg.abs().mean(1, keepdim=True) * (1 + n.square()))
        check(grads.x, want, slack, of)
        check(grads.norm_weight, (dx * n).sum(0), (err * n.abs()).sum(0) + (B + 8) * U * (dx * n).abs().sum(0), torch.float32)
        check(grads.norm_bias, dx.sum(0), err.sum(0) + (B + 8) * U * dx.abs().sum(0), torch.float32)
    again = layer.backward(s, dout, dx_dtype=dtype)
    for a, b in zip(grads, again):
        assert (a is None and b is None) or torch.equal(a, b)


def test_refusals(device):
    layer = layer_of(4, 128, 64, 32, 2, device)
    _, s = layer.forward(torch.zeros(3, 128, device=device))
    for bad in (FP8, torch.float64, torch.int32):
        with pytest.raises(ValueError):
            layer.backward(s, torch.zeros(3, 32, device=device), dx_dtype=bad)
