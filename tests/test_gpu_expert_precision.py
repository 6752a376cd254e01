"""What eb_expert_product's sums hold: exact outputs, sums that cancel, single large products among
small ones, in every size of tile.

Sizes are given as slots and weight rows; 16-bit outputs of these take, in this order, the stream
kernel and the tiles of 32, 64, 128 and 256 slots.
"""
import pytest
import torch

from paper_2512_05831_amd import experts as ex

pytestmark = pytest.mark.gpu
SIZES = [(40, 200), (300, 1000), (2048, 1664), (2048, 4096), (8192, 4100)]
FP8 = torch.float8_e4m3fn


def integers(rows, cols, gen, device):
    return torch.randint(-4, 5, (rows, cols), generator=gen).float().to(device)


def unit_scales(M, N, K, device):
    kb = -(-K // 128)
    return torch.ones(kb, M, device=device).t(), torch.ones(-(-N // 128), kb, device=device)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_RELU])
def test_large_products_among_small_ones(dtype, M, N, act, device):
    """Integers, of which two large products in a block cancel: every sum is below 2^24 and exact in fp32.  With
    EB_EXACT_SUMS so is the output before its one rounding; without it a 16-bit output is off by less than 2^-10 of the
    largest of each eight products."""
    K = 384
    g = torch.Generator().manual_seed(M)
    x, w = integers(M, K, g, device), integers(N, K, g, device)
    x[:, 128 + 40], x[:, 128 + 43] = 448, 448
    w[:, 128 + 40], w[:, 128 + 43] = 448, -448
    xs, ws = unit_scales(M, N, K, device)
    exact = x.double() @ w.double().t()
    exact = exact.clamp(min=0) if act == ex.EB_ACT_RELU else exact
    call = lambda a, **kw: ex.product(x.to(FP8), xs, w.to(FP8), ws, act=a, **kw)  # noqa: E731
    assert torch.equal(call(act | ex.EB_EXACT_SUMS, out_dtype=dtype), exact.to(dtype))
    wide = torch.full((M, N + 9), 7.0, dtype=dtype, device=device)  # rows that start anywhere
    call(act | ex.EB_EXACT_SUMS, out=wide[:, 5:5 + N])
    assert torch.equal(wide[:, 5:5 + N], exact.to(dtype)) and (wide[:, :5] == 7.0).all() and (wide[:, 5 + N:] == 7.0).all()
    off = (call(act, out_dtype=dtype).double() - exact).abs()
    assert (off <= 448.0 ** 2 * 2.0 ** -10 * (1 + 2.0 ** -8) + 2.0 ** -8 * exact.abs()).all()
