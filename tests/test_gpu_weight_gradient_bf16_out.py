"""bfloat16 outputs of eb_weight_gradient: products within 2^-16 of exact (where two parts of bfloat16 hold a scaled value: 2^-17,
the first part being off by at most half a step of 8 bits, which the second holds in 8 bits again), rounded once."""
import pytest

from paper_2512_05831_amd import train
from train_util import U, check
from test_gpu_weight_gradient import BF16, TYPES, operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", TYPES)
def test_sums_of_bfloat16_outputs(types, device):
    """As exact as others' but for the output's rounding: sums that cancel show what products lost."""
    for M, K in ((300, 256), (3000, 130)):
        dy, x = operands(M, M, 140, K, *types, device)
        got = train.weight_gradient(dy[0], x[0], dy_scales=dy[1], x_scales=x[1], out_dtype=BF16)
        want, size = dy[2].t() @ x[2], dy[2].abs().t() @ x[2].abs()
        check(got, want, (2.0 ** -17 + (M + 40) * U) * size, BF16)
