"""eb_layer_norm_backward where its sums over the rows have more columns than one launch of a workgroup per 64 holds."""
import pytest
import torch

from paper_2512_05831_amd import train
from train_util import U

pytestmark = pytest.mark.gpu


def test_more_columns_than_one_launch_joins(device):
    cols = (1 << 27) + 72
    g = torch.Generator(device=device).manual_seed(1)
    dy, x = (torch.randn(2, cols, generator=g, device=device, dtype=torch.bfloat16) for _ in range(2))
    rstd, mean = torch.tensor([0.5, 2.0], device=device), torch.tensor([0.25, -1.0], device=device)
    dx, dw, db = train.layer_norm_backward(dy, x, rstd, mean=mean)
    for lo in range(0, cols, 1 << 25):
        d, v = (t[:, lo:lo + (1 << 25)].double() for t in (dy, x))
        n = (v - mean.double()[:, None]) * rstd.double()[:, None]
        each = (d * n).abs().sum(0)
        # three roundings of n, one of the product, two additions (a join's zeros add nothing)
        assert ((dw[lo:lo + (1 << 25)].double() - (d * n).sum(0)).abs() <= 8 * U * each + 2.0 ** -140).all()
        assert ((db[lo:lo + (1 << 25)].double() - d.sum(0)).abs() <= 2 * U * d.abs().sum(0)).all()
    assert dx.shape == dy.shape and bool(dx.isfinite().all())
