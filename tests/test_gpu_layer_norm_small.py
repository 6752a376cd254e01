"""eb_layer_norm of rows whose centred values lie below what a factor of 448 / largest can be made of (448 x 2^-126): what is kept in
8 bits has its scale from the normalised values, above that."""
import pytest
import torch

from paper_2512_05831_amd import train
from train_util import FP8, check8, generator
from test_gpu_layer_norm import forward

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -149


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(5, 300), (5, 304), (2100, 304), (3, 5000), (4, 20000)])
def test_layer_norm_of_small_rows(rows, cols, dtype, device):
    """Rows of 1e-39 and up, centred below the floor; rstd (1e-5 under the root: 316) lifts them over it."""
    sizes = torch.tensor([1e-38, 3e-39, 1e-37, 3e-36, 1.0], device=device).repeat(rows // 5 + 1)[:rows]
    x = (torch.rand(rows, cols, generator=generator(device, cols), device=device) * sizes[:, None]).to(dtype)
    w, b = torch.ones(cols, device=device), torch.zeros(cols, device=device)
    r = train.layer_norm(x, w, b, checkpoint=True, out_dtype=FP8)
    _, (rstd, _), (n, en), (y, ey) = forward(x.double(), w, b, 1e-5)
    # A mean, and its difference to a value, are rounded to a multiple of 2^-149, as n and y are; a difference below the
    # smallest normal number once more in the product's factors.
    en, ey = (e + 4 * LEAST * rstd + 2 * LEAST for e in (en, ey))
    check8(r.kept, r.kept_scales, n, en)
    check8(r.y, r.y_scales, y, ey)
