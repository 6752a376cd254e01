"""GPU parity of eb_dispatch, eb_combine and eb_combine_backward with their formulas in 64 bits.

A joined value is K products and additions: (K + 1) u of the sum of their sizes (u =
2^-24), and the rounding to its type; a gradient of y is one product; a gradient of a
weight passes 8 additions for each 512 columns and 10 more.
"""
import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex, train
from train_util import EVERY_REMAINDER, FP8, U, WIDE, among_nans, as_type, check, check8, generator, route_of

pytestmark = pytest.mark.gpu
WIDTHS = [1, 3, 8, 16, 31, 64, 100, 128, 129, 512, 513, 1000, 1024, 1512, 2048, 2100, 4096, 5000]


def bits(x):
    return x.contiguous().view(torch.uint8)


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dtype", WIDE + [FP8])
def test_dispatch(cols, dtype, device):
    r = route_of(37, 6, 3, device, cols, shards=2)
    x, s, _ = as_type(torch.randn(37, cols, generator=generator(device, cols), device=device), dtype)
    used = int(r.offsets[-1])
    if dtype == FP8:
        got, scales = train.dispatch(x, r.tokens, s)
        assert torch.equal(scales[:used], s[r.tokens[:used].long()])
    else:
        room = torch.full((111, cols + 3), 5.0, device=device).to(dtype)
        got = train.dispatch(x, r.tokens, out=room[:, 1:cols + 1])
        assert (got[used:] == 5).all() and (room[:, 0] == 5).all() and (room[:, cols + 1:] == 5).all()
        assert torch.equal(bits(train.dispatch(x, r.tokens)[:used]), bits(got[:used]))
    assert 0 < used < 111 and torch.equal(bits(got[:used]), bits(x[r.tokens[:used].long()]))


def test_dispatch_odd_places(device):
    """Views, tokens out of range, the same token again, one slot, none."""
    x = torch.randn(20, 300, generator=generator(device, 1), device=device).to(torch.bfloat16)
    tokens = torch.tensor([3, 3, -1, 19, 20, -2147483648, 2147483647, 0, 3], dtype=torch.int32, device=device)
    for view in (x[:, 7:], x[:, 1:9], x[:, 2:3], x):
        out = torch.zeros(9, view.shape[1], dtype=x.dtype, device=device)
        train.dispatch(view, tokens, out=out)
        ok = (tokens >= 0) & (tokens < 20)
        assert torch.equal(out[ok], view[tokens[ok].long()]) and (out[~ok] == 0).all()
    assert torch.equal(train.dispatch(x, tokens[3:4]), x[19:20])
    assert train.dispatch(x, tokens[:0]).shape == (0, 300)
    out = torch.ones(9, 300, dtype=x.dtype, device=device)
    assert (train.dispatch(x[:0], tokens, out=out) == 1).all()


def joined(y, slots, w):
    ok = (slots >= 0) & (slots < y.shape[0])
    rows = torch.where(ok[:, :, None], y.double()[slots.clamp(0, max(0, y.shape[0] - 1)).long()], 0.0)
    if w is not None:
        rows = rows * w.double()[:, :, None]
    return rows.sum(1), (slots.shape[1] + 1) * U * rows.abs().sum(1)


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dtype", WIDE)
def test_combine(cols, dtype, device):
    for N, E, top, shards in ((41, 9, 5, 1), (3, 4, 1, 2), (10, 64, 64, 1)):
        r = route_of(N, E, top, device, cols + top, shards)
        y = torch.randn(N * top, cols, generator=generator(device, cols), device=device).to(dtype)
        for out in WIDE:
            check(train.combine(y, r.slots, r.weights, out_dtype=out), *joined(y, r.slots, r.weights), out)
        check(train.combine(y, r.slots), *joined(y, r.slots, None), dtype)


def test_combine_odd_places(device):
    """Tokens without pairs, slots out of range, the same slot again, views; NaNs that no pair names stay out."""
    y = torch.randn(9, 77, generator=generator(device, 1), device=device)
    y[4] = float("nan")
    slots = torch.tensor([[-1, -1], [0, 0], [8, 9], [-5, 2147483647], [-2147483648, 3], [1, 2]], dtype=torch.int32, device=device)
    w = torch.tensor([[1.0, 2.0], [0.5, 0.25], [0.0, 7.0], [1.0, float("nan")], [float("inf"), 2.0], [-1.0, 1.0]], device=device)
    got = train.combine(y[:, 3:], slots, w)
    assert (got[0] == 0).all() and (got[3] == 0).all()
    check(got, *joined(y[:, 3:], slots, torch.where((slots >= 0) & (slots < 9), w, 0.0)), torch.float32)
    assert train.combine(y, slots[:0]).shape == (0, 77)
    assert (train.combine(y[:0], slots, w) == 0).all()


def gradients(dout, y, slots, w):
    N, K = slots.shape
    ok = (slots >= 0) & (slots < y.shape[0])
    at = slots.clamp(0, max(0, y.shape[0] - 1)).long()
    dots = dout.double()[:, None] * y.double()[at]
    h = 8 * -(-y.shape[1] // 512) + 10
    dw, edw = torch.where(ok, dots.sum(2), 0.0), torch.where(ok, h * U * dots.abs().sum(2), 0.0)
    rows = dout.double()[:, None] * (torch.ones_like(slots) if w is None else w).double()[:, :, None]
    return rows[ok], at[ok], dw, edw


def check_gradients(dout, y, r_slots, w, out):
    rows, at, dw, edw = gradients(dout, y, r_slots, w)
    got = train.combine_backward(dout, y, r_slots, w, out_dtype=out)
    check(got.dweights, dw, edw, torch.float32)
    assert got.dy.shape == y.shape
    if out == FP8:
        pitch = got.dy.stride(0)
        padded = got.dy.as_strided((y.shape[0], pitch), (pitch, 1))[at][:, :y.shape[1]]
        check8(padded, got.dy_scales[at], rows, U * rows.abs())
        if pitch > y.shape[1]:
            whole = got.dy.as_strided((y.shape[0], pitch), (pitch, 1)).view(torch.uint8)
            assert (whole[at][:, y.shape[1]:] == 0).all()
    else:
        check(got.dy[at], rows, U * rows.abs(), out)


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dout_type,y_type", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)])
def test_combine_backward(cols, dout_type, y_type, device):
    for N, E, top, shards in ((41, 9, 5, 1), (3, 4, 1, 2), (10, 64, 64, 1)):
        r = route_of(N, E, top, device, cols + top, shards)
        g = generator(device, cols)
        y = torch.randn(N * top, cols, generator=g, device=device).to(y_type)
        dout = torch.randn(N, cols, generator=g, device=device).to(dout_type)
        for out in (FP8, torch.bfloat16, torch.float32, torch.float16):
            check_gradients(dout, y, r.slots, r.weights, out)
        check_gradients(dout, y, r.slots, None, FP8)


def test_combine_backward_odd_places(device):
    """Rows that are no pair's slot stay as they were; weights of 0, infinity and NaN; no tokens."""
    g = generator(device, 2)
    y, dout = torch.randn(9, 300, generator=g, device=device), torch.randn(4, 300, generator=g, device=device)
    slots = torch.tensor([[0, -1], [8, 2], [9, -7], [5, 4]], dtype=torch.int32, device=device)
    w = torch.tensor([[0.0, 1.0], [-2.0, float("nan")], [1.0, 1.0], [float("inf"), 0.5]], device=device)
    dw = torch.empty(4, 2, device=device)
    dy = torch.full((9, 300), 7.0, device=device)
    train.eb_combine_backward(4, 2, 300, dout.data_ptr(), eb.EB_F32, 300, y.data_ptr(), eb.EB_F32, 300, 9, slots.data_ptr(), w.data_ptr(),
                              eb.EB_F32, dy.data_ptr(), 300, None, 0, dw.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert (dy[[1, 3, 6, 7]] == 7).all() and (dy[0] == 0).all() and dy[2].isnan().all() and dy[5].isinf().all()
    assert torch.equal(dy[8], -2 * dout[1]) and torch.equal(dy[4], 0.5 * dout[3])
    _, _, want, err = gradients(dout, y, slots, w)
    check(dw, want, err, torch.float32)
    got = train.combine_backward(dout, y, slots, w, out_dtype=FP8)
    assert got.dy_scales[2].isnan().all() and got.dy[2].float().isnan().all() and got.dy_scales[5].isnan().all()
    assert train.combine_backward(dout[:0], y, slots[:0]).dweights.shape == (0, 2)
    only = torch.full((4, 2), -1.0, device=device)  # without dy, and without dweights
    args = (4, 2, 300, dout.data_ptr(), eb.EB_F32, 300, y.data_ptr(), eb.EB_F32, 300, 9, slots.data_ptr(), w.data_ptr(), eb.EB_F32)
    train.eb_combine_backward(*args, None, 0, None, 0, only.data_ptr(), None)
    torch.cuda.synchronize()
    assert torch.equal(only, dw)
    dy.fill_(7.0)
    train.eb_combine_backward(4, 2, 300, dout.data_ptr(), eb.EB_F32, 300, None, eb.EB_F32, 300, 9, slots.data_ptr(), w.data_ptr(), eb.EB_F32,
                              dy.data_ptr(), 300, None, 0, None, None)
    torch.cuda.synchronize()
    assert torch.equal(dy[8], -2 * dout[1])


def test_sorted_and_joined_is_the_identity(device):
    """One GPU's pairs, every weight 1 / top: what is dispatched comes back."""
    r = route_of(500, 16, 4, device, 3)
    x = torch.randn(500, 512, generator=generator(device, 4), device=device).to(torch.bfloat16)
    back = train.combine(train.dispatch(x, r.tokens), r.slots, torch.full((500, 4), 0.25, device=device))
    assert torch.equal(back, x)


def test_row_offsets_past_32_bits(device):
    y = torch.empty(3, 1 << 30, dtype=torch.float16, device=device)
    y[:, :200] = torch.randn(3, 200, generator=generator(device, 4), device=device).to(torch.float16)
    tokens = torch.tensor([2, 0, 1], dtype=torch.int32, device=device)
    assert torch.equal(train.dispatch(y[:, :200], tokens), y[:, :200][tokens.long()])
    slots = tokens.view(3, 1)
    assert torch.equal(train.combine(y[:, :200], slots), y[:, :200][tokens.long()])


def test_refusals(device):
    x = torch.zeros(4, 32, device=device)
    q, s = ex.quantize_fp8(x)
    i = torch.zeros(4, dtype=torch.int32, device=device)
    slots = i.view(2, 2)
    w = torch.ones(2, 2, device=device)
    for bad in (lambda: train.dispatch(x, i.long()), lambda: train.dispatch(x, i[::2]), lambda: train.dispatch(x, i.cpu()), lambda: train.dispatch(q, i),
                lambda: train.dispatch(x, i, out=x.half()), lambda: train.dispatch(x, i, out=x[:3]), lambda: train.dispatch(q, i, s, out=q),
                lambda: train.dispatch(x.t(), i), lambda: train.combine(q, slots), lambda: train.combine(x, i), lambda: train.combine(x, slots, w[:1]),
                lambda: train.combine(x, slots, w.double()), lambda: train.combine(x, slots.long()), lambda: train.combine(x, slots, out_dtype=FP8),
                lambda: train.combine_backward(x[:2], x[:, :31], slots), lambda: train.combine_backward(x, x, slots),
                lambda: train.combine_backward(x[:2], q, slots), lambda: train.combine_backward(x[:2], x.cpu(), slots),
                lambda: train.combine_backward(x[:2], x, slots, w.cpu())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(eb.EbError) as e:
        train.combine(x, torch.zeros(2, 65, dtype=torch.int32, device=device))
    assert e.value.code == eb.EB_ERR_UNSUPPORTED


@pytest.mark.parametrize("cols", EVERY_REMAINDER)
@pytest.mark.parametrize("dtype", WIDE)
def test_every_remainder(cols, dtype, device):
    """Rows that end anywhere in a chunk of 8, with NaN before and behind them."""
    r = route_of(13, 6, 3, device, cols)
    g = generator(device, cols)
    y = among_nans(torch.randn(39, cols, generator=g, device=device).to(dtype))
    dout = among_nans(torch.randn(13, cols, generator=g, device=device).to(dtype))
    check(train.combine(y, r.slots, r.weights, out_dtype=dtype), *joined(y, r.slots, r.weights), dtype)
    for out in (FP8, dtype):
        check_gradients(dout, y, r.slots, r.weights, out)
