"""Arguments of the experts' wrappers and of ``ExpertLayer``: calls without work, shapes
that do not fit, streams and devices.
"""
import contextlib

import pytest
import torch

from paper_2512_05831_amd import experts as ex
from test_gpu_expert_layer import layer_of
from test_gpu_expert_product import Case, blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shape", [(3, 0, 200), (0, 5, 200), (0, 0, 16), (2, 0, 1)])
def test_stacks_without_rows(shape, block_rows, device):
    q, s = ex.quantize_fp8(torch.empty(shape, device=device), block_rows=block_rows)
    m, rows, cols = shape
    assert q.shape == shape and q.dtype == torch.float8_e4m3fn
    assert s.shape == (m, rows if block_rows == 1 else blocks(rows), blocks(cols))


@pytest.mark.parametrize("E", [1, 3])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_SILU_GATE])
def test_scales_and_bias_of_another_shape(E, act, device):
    """As many values in another order: a transposed matrix of scales, a bias by output, then expert."""
    case = Case(40, 300, 600, device, E=E, act=act, bias=True, counts=[40 // E + (e < 40 % E) for e in range(E)])
    want = case.run(out_dtype=torch.float32)
    good, bias = case.ws, case.bias
    for same in (good.clone(), good.view(E, -1, good.shape[-2], good.shape[-1])) + ((good[0],) if E == 1 else ()):
        case.ws = same
        assert torch.equal(case.run(out_dtype=torch.float32), want)
    if act == ex.EB_ACT_SILU_GATE:  # as the halves' own matrices
        case.ws = good.view(2 * E, -1, good.shape[-1])
        assert torch.equal(case.run(out_dtype=torch.float32), want)
    for bad in (good.transpose(-1, -2).contiguous(), good.flatten(), good.reshape(1, -1), good.reshape(-1, 1)):
        case.ws = bad
        with pytest.raises(ValueError):
            case.run(out_dtype=torch.float32)
    case.ws = good
    for bad in (bias.t().contiguous(), bias.reshape(-1, 1)) + ((bias.flatten(),) if E > 1 else ()):
        case.bias = bad
        with pytest.raises(ValueError):
            case.run(out_dtype=torch.float32)
    case.bias = bias[0] if E == 1 else bias
    assert torch.equal(case.run(out_dtype=torch.float32), want)


def test_out_of_another_type_than_asked_for(device):
    case = Case(8, 64, 128, device)
    out = torch.empty(8, 64, dtype=torch.bfloat16, device=device)
    for dtype in (torch.float32, torch.float16, torch.float8_e4m3fn):
        with pytest.raises(ValueError):
            case.run(out=out, out_dtype=dtype)
    assert torch.equal(case.run(out=out, out_dtype=torch.bfloat16), case.run())


def test_layer_refuses_scores_of_another_shape(device):
    layer = layer_of(8, 256, 128, 64, 2, ex.EB_ACT_RELU, device)
    x = torch.randn(10, 256, device=device)
    layer.forward(x, torch.zeros(10, 8, device=device))
    for scores in (torch.zeros(9, 8, device=device), torch.zeros(11, 8, device=device), torch.zeros(10, 9, device=device), torch.zeros(80, device=device)):
        with pytest.raises(ValueError):
            layer.forward(x, scores)
    for bad in (x[:, :200], x[0], x.view(2, 5, 256)):
        with pytest.raises(ValueError):
            layer.forward(bad, torch.zeros(bad.shape[0], 8, device=device))


class Entered:
    """Stands for torch.cuda.device: notes which GPU is made current."""

    def __init__(self):
        self.devices = []

    def __call__(self, device):
        self.devices.append(device.index)
        return contextlib.nullcontext()


def test_calls_go_to_the_tensors_gpu(device, monkeypatch):
    """With another GPU current the tensors' own is made so: the default stream is the current GPU's."""
    case = Case(8, 64, 128, device)
    layer = layer_of(8, 256, 128, 64, 2, ex.EB_ACT_RELU, device)
    x, scores = torch.randn(4, 256, device=device), torch.randn(4, 8, device=device)
    want = case.run(), ex.quantize_fp8(x), ex.route(scores, 2), layer.forward(x, scores)
    entered = Entered()
    monkeypatch.setattr(torch.cuda, "device", entered)
    calls = (lambda: case.run(), lambda: ex.quantize_fp8(x), lambda: ex.route(scores, 2), lambda: layer.forward(x, scores))
    for call in calls:
        call()
    assert entered.devices == []  # this GPU is current
    monkeypatch.setattr(ex, "_gpu", lambda: device.index + 1)
    for call, result in zip(calls, want):
        entered.devices.clear()
        got = call()
        assert entered.devices and set(entered.devices) == {device.index}
        for a, b in zip(got if isinstance(got, tuple) else (got,), result if isinstance(result, tuple) else (result,)):
            assert torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a, b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)


def test_layer_without_tokens(device):
    layer = layer_of(8, 256, 128, 64, 2, ex.EB_ACT_SILU_GATE, device)
    assert layer.forward(torch.empty(0, 256, device=device)).shape == (0, 64)


@pytest.mark.parametrize("M", [30, 3000])
def test_product_and_quantize_on_another_stream(M, device):
    """The stream that is given carries the call: what it has to wait for is written there just before."""
    case = Case(M, 512, 700, device, E=3, act=ex.EB_ACT_SILU_GATE, counts=[M // 3, 1, M - M // 3 - 1], gather=200)
    x = torch.randn(M, 700, device=device)
    want, want8, wantq = case.run(), case.run(out_dtype=torch.float8_e4m3fn), ex.quantize_fp8(x)
    wantw = ex.quantize_fp8(x, block_rows=128)
    held, scales, values = case.x.clone(), case.xs.t().contiguous().t(), x.clone()
    pitched = torch.zeros(held.shape[0], 704, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)[:, :700]
    late_x, late_s, late_v = pitched, torch.zeros_like(case.xs.t().contiguous()).t(), torch.zeros_like(x)
    big = torch.randn(4096, 4096, device=device)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):  # holds the side stream back
            big = big @ big * 1e-3
        late_x.view(torch.uint8).copy_(held.view(torch.uint8))
        late_s.copy_(scales)
        late_v.copy_(values)
    case.x, case.xs = late_x, late_s
    got, got8 = case.run(stream=side), case.run(out_dtype=torch.float8_e4m3fn, stream=side)
    gotq, gotw = ex.quantize_fp8(late_v, stream=side), ex.quantize_fp8(late_v, block_rows=128, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    for mine, other in ((got8, want8), (gotq, wantq), (gotw, wantw)):
        assert torch.equal(mine[0].view(torch.uint8), other[0].view(torch.uint8)) and torch.equal(mine[1], other[1])


def test_an_older_error_is_not_the_calls(device):
    """An error that another call left with the runtime on this thread is not reported as the route's."""
    from paper_2512_05831_amd import eb

    runtime = eb.library()  # its runtime's functions are found through it
    x = torch.empty(0, 32, device=device)
    ex.route(x, 4)
    assert runtime.hipSetDevice(1 << 20) != 0
    try:
        r = ex.route(x, 4, shard_lo=8, shard_hi=24)
    finally:
        runtime.hipGetLastError()
    assert r.offsets.tolist() == [0] * 17
