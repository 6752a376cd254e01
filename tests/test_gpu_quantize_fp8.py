"""GPU parity of eb_quantize_fp8 with its definition.

The scale is a single fp32 division, so the CPU's gives the same bits.  The
exact quotient x * 448 / most is rounded to nearest even: x * 448 and the
middles of e4m3 numbers times most are compared in 64 bits, which hold both, so
that gives the same bits too.  And |q * scale - x| <= |x| 2^-4 (1 + 2^-20) +
scale * 2^-10 (half a step of e4m3, normal and subnormal, and the rounding of
the scale).
"""
import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex

pytestmark = pytest.mark.gpu
INF = float("inf")


def plain(x, block_rows):
    """q and scales of [m, rows, cols], on the CPU."""
    m, rows, cols = x.shape
    rb, cb = -(-rows // block_rows), -(-cols // 128)
    full = torch.zeros(m, rb * block_rows, cb * 128)
    full[:, :rows, :cols] = x.float()
    b = full.view(m, rb, block_rows, cb, 128)
    most = b.abs().amax((2, 4))
    s = torch.where(torch.isfinite(most), (most / 448).clamp(min=2.0 ** -126), float("nan"))
    at = most.double().clamp(min=448 * 2.0 ** -126)[:, :, None, :, None]
    x448 = b.double().abs() * 448
    step = torch.exp2(torch.floor(torch.log2((x448 / at).clamp(min=2.0 ** -6))) - 3)
    k = torch.floor(x448 / at / step)
    middle = (k + 0.5) * step * at
    k += (x448 > middle) | ((x448 == middle) & (k % 2 == 1))
    q = torch.where(s.isnan()[:, :, None, :, None], float("nan"), torch.copysign(k * step, b.double()))
    return q.view(m, rb * block_rows, cb * 128)[:, :rows, :cols].to(torch.float8_e4m3fn), s


def bits(q):
    return q.contiguous().view(torch.uint8)


def check(x, block_rows, device):
    dev = x.to(device) if not x.is_cuda else x
    q, s = ex.quantize_fp8(dev, block_rows=block_rows)
    x3 = x.cpu() if x.dim() == 3 else x.cpu()[None]
    want_q, want_s = plain(x3, block_rows)
    q3, s3 = (q.cpu(), s.cpu()) if x.dim() == 3 else (q.cpu()[None], s.cpu()[None])
    assert torch.equal(s3.nan_to_num(nan=-1.0), want_s.nan_to_num(nan=-1.0))
    nan = want_q.float().isnan()
    assert torch.equal(q3.float().isnan(), nan)
    assert torch.equal(bits(q3)[~nan], bits(want_q)[~nan])
    if not nan.any():
        each = s3.double().repeat_interleave(block_rows, 1)[:, :x3.shape[1]].repeat_interleave(128, 2)[:, :, :x3.shape[2]]
        off = (q3.double() * each - x3.double()).abs()
        assert (off <= x3.double().abs() * 2.0 ** -4 * (1 + 2.0 ** -20) + each * 2.0 ** -10).all()
    # The bytes between the columns and the next multiple of 16 are zeros.
    cols, pitch = q.shape[-1], q.stride(-2)
    if pitch > cols and q.shape[-2] > 0:
        rows = q.shape[0] * q.shape[1] if q.dim() == 3 else q.shape[0]
        whole = q.as_strided((rows, pitch), (pitch, 1))
        assert (bits(whole)[:, cols:] == 0).all()
    return q, s


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 127), (3, 128), (17, 129), (16, 512), (33, 189), (5, 1000), (250, 1512), (64, 3328), (1000, 77)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_matrix(dtype, rows, cols, block_rows, device):
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g) * torch.rand(rows, 1, generator=g).mul(8).exp2()
    check(x.to(dtype), block_rows, device)


@pytest.mark.parametrize("m,rows,cols", [(3, 128, 256), (5, 200, 70), (2, 1, 300), (4, 129, 1024)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_stacked_matrices(m, rows, cols, block_rows, device):
    check(torch.randn(m, rows, cols, generator=torch.Generator().manual_seed(m)), block_rows, device)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_and_odd_addresses(block_rows, dtype, device):
    big = torch.randn(90, 700, device=device).to(dtype)
    for view in (big[3:80, 5:500], big[::2, 1:600], big[:, 8:520], big[7:8, 3:40]):
        check(view, block_rows, device)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_extremes(block_rows, device):
    x = torch.randn(300, 400, generator=torch.Generator().manual_seed(1))
    x[0] = 0
    x[1] *= 1e-38
    x[2] *= 1e-42
    x[3] = torch.finfo(torch.float32).max
    x[4, ::7] = torch.finfo(torch.float32).min
    x[5, 13] = INF
    x[140, 399] = -INF
    x[7, 130] = float("nan")
    x[299, 399] = float("nan")
    x[9] = torch.arange(400) % 449  # every integer up to 448, halfway cases among them
    x[10] = -0.0
    check(x, block_rows, device)


def test_rounds_to_nearest_even(device):
    """Every e4m3 number, and the points halfway between neighbours, under the scale 1."""
    values = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()  # 0 .. 448
    half = (values[1:] + values[:-1]) / 2
    x = torch.zeros(2, 128)
    x[0, :127] = values
    x[1, :126] = half
    x[1, 127] = 448.0
    q, s = check(torch.cat([x, -x]), 1, device)
    assert (s == 1).all()
    assert torch.equal(q[0, :127].float().cpu(), values)


def test_no_rows(device):
    q, s = ex.quantize_fp8(torch.empty(0, 200, device=device))
    assert q.shape == (0, 200) and s.shape == (0, 2)


def test_row_offsets_past_32_bits(device):
    """Rows far apart: byte offsets of x past 2^32."""
    big = torch.empty(5, 1 << 29, dtype=torch.bfloat16, device=device)
    big[:, :300] = torch.randn(5, 300, device=device).to(torch.bfloat16)
    check(big[:, :300], 1, device)
    check(big[:, :300], 128, device)


def test_refusals(device):
    x = torch.zeros(4, 32, device=device)
    with pytest.raises(eb.EbError) as e:
        ex.quantize_fp8(x, block_rows=64)
    assert e.value.code == eb.EB_ERR_INVALID
    for bad in (x.double(), x.cpu(), x.t(), x[0], torch.zeros(6, 4, 32, device=device)[::2]):
        with pytest.raises(ValueError):
            ex.quantize_fp8(bad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quotients_at_and_by_the_middle(dtype, block_rows, device):
    """Values at the exact middles of e4m3 numbers times most / 448, and their neighbours, at every size."""
    values = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    middle = (values[1:] + values[:-1]) / 2
    tiny, huge = torch.finfo(dtype).tiny, torch.finfo(dtype).max
    rows = []
    for most in (448.0, 1.0, 7.0, 3.5, 0.4375, 1.75 * 2.0 ** 9, 5.0, 1.1, huge, huge / 2, tiny * 448, tiny * 460, tiny * 512):
        x = (middle * (most / 448)).to(dtype)
        for y in (x, torch.nextafter(x, torch.zeros_like(x)), torch.nextafter(x, torch.full_like(x, INF))):
            row = torch.zeros(128, dtype=dtype)
            row[:126] = torch.where(y.float().abs() > most, torch.zeros_like(y), y)
            row[1:126:2] *= -1
            row[127] = most
            rows.append(row)
    x = torch.stack(rows)
    check(x, 1, device) if block_rows == 1 else [check(r.expand(3, 128).contiguous(), 128, device) for r in rows]
