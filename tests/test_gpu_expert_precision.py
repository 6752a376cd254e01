"""What eb_expert_product's sums hold: exact outputs, sums that cancel, single large products among
small ones, in every size of tile.

Sizes are given as slots and weight rows; 16-bit outputs of these take, in this order, the stream
kernel and the tiles of 32, 64, 128 and 256 slots.
"""
import pytest
import torch

from paper_2512_05831_amd import experts as ex
from test_gpu_expert_layer import layer_of

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


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("K", [640, 3328, 1000])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_RELU])
def test_small_integers_are_rounded_once(dtype, M, N, K, act, device):
    """Products below 2^5 and sums below 2^17: exact in either matrix unit, then one rounding."""
    g = torch.Generator().manual_seed(M + K)
    pitch = -(-K // 16) * 16
    x, w = integers(M, pitch, g, device), integers(N, pitch, g, device)
    xs, ws = unit_scales(M, N, K, device)
    got = ex.product(x.to(FP8)[:, :K], xs * 0.5, w.to(FP8)[:, :K], ws * 4.0, act=act, out_dtype=dtype)
    want = 2 * x[:, :K].double() @ w[:, :K].double().t()
    want = want.clamp(min=0) if act == ex.EB_ACT_RELU else want
    assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,N", SIZES)
def test_sums_that_cancel(dtype, M, N, device):
    """Two blocks of 128 whose exact sums are each other's opposite, their inputs in another order: what is left is
    the two sums' error, each at most 1.5e-5 (and a tenth) of the sums' root mean square."""
    g = torch.Generator().manual_seed(N)
    draw = lambda rows: (torch.randn(rows, 128, generator=g) * 100).clamp(-448, 448).to(FP8).float().to(device)  # noqa: E731
    x, w, order = draw(M), draw(N), torch.randperm(128, generator=g).to(device)
    xs, ws = unit_scales(M, N, 256, device)
    scale = 2.0 ** -10  # keeps fp16 from its ends
    got = ex.product(torch.cat([x, x[:, order]], 1).to(FP8), xs * scale, torch.cat([w, -w[:, order]], 1).to(FP8), ws, out_dtype=dtype)
    rms = (x.double() @ w.double().t()).pow(2).mean().sqrt() * scale
    assert got.double().pow(2).mean().sqrt() <= 2 * 1.1 * 1.5e-5 * rms


@pytest.mark.parametrize("M", [16, 400, 20000])
def test_gate_over_its_range(M, device):
    """g / (1 + exp(-g)) for any g: one input under a scale, and a bias of 1 for what is gated.  Within 4 + |g| ulp, or
    2^-119 (a reciprocal below fp32's normal numbers)."""
    N = 256
    g = torch.linspace(-130, 130, M, device=device)
    g[: M // 4] = torch.linspace(-4, 4, M // 4, device=device)
    w = torch.zeros(N, 16, device=device)
    w[: N // 2, 0] = 1.0
    x = torch.zeros(M, 16, device=device)
    x[:, 0] = 1.0
    bias = torch.zeros(N, device=device)
    bias[N // 2:] = 1.0
    y = ex.product(x.to(FP8), g[:, None], w.to(FP8), torch.ones(2, 1, device=device), bias=bias, act=ex.EB_ACT_SILU_GATE, out_dtype=torch.float32)
    d = g.double()
    want = (d * torch.sigmoid(d))[:, None]
    assert ((y.double() - want).abs() <= (4 + d.abs()[:, None]) * 2.0 ** -23 * want.abs() + 2.0 ** -119).all()


@pytest.mark.parametrize("rows", [None, torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("exact", [0, ex.EB_EXACT_SUMS])
@pytest.mark.parametrize("B", [5, 1500])
def test_layer_joins_rows_of_the_type_asked_for(rows, exact, B, device):
    """The layer's result is the weighted sum of the second product's rows in that type: top products and sums in fp32."""
    top = 3
    g = torch.Generator(device=device).manual_seed(B)
    w_up, w_down, router, x, scores = (torch.randn(*n, generator=g, device=device) for n in ((8, 768, 256), (8, 200, 384), (8, 256), (B, 256), (B, 8)))
    layer = ex.ExpertLayer(w_up / 16, w_down / 16, router, top, act=ex.EB_ACT_SILU_GATE | exact, row_dtype=rows)
    r = ex.route(scores, top)
    h, hs = ex.product(*ex.quantize_fp8(x), layer.w_up, layer.up_scales, r.offsets, r.tokens, act=ex.EB_ACT_SILU_GATE, out_dtype=FP8)
    y = ex.product(h, hs, layer.w_down, layer.down_scales, r.offsets, act=exact, out_dtype=rows or torch.bfloat16).double()
    each = y[r.slots.long()] * r.weights.double()[:, :, None]
    off = (layer.forward(x, scores).double() - each.sum(1)).abs()
    assert (off <= 2 * top * 2.0 ** -24 * each.abs().sum(1)).all()


def test_layer_refuses_rows_of_other_types(device):
    for rows in (FP8, torch.float64, torch.int32):
        with pytest.raises(ValueError):
            layer_of(2, 16, 16, 16, 1, ex.EB_ACT_RELU, device, row_dtype=rows)
