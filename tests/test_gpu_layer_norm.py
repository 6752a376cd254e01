"""GPU parity of eb_layer_norm and eb_layer_norm_backward with their formulas in 64 bits.

With u = 2^-24 and h the additions that a value passes on its way into a row's sum
(8 of each 512 columns in a lane, then 12 over lanes and waves), a mean errs by
em = h u mean|x| + u|m|.  The centred squares then hold var + em^2, with h + 6
roundings; r = 1 / sqrt errs by half of that and 2 u.  n = (x - m) r: |n| (er + 3 u) +
em r;  y = n w + b: |w| en + 2 u (|n w| + |b|).  The backward pass has n from given
statistics (3 u |n|) or held in 8 bits (u |n|), and sums of h roundings again; the sums
over rows pass at most min(rows, rows / 512 + 140) + 4 additions.
"""
import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex, train
from train_util import EVERY_REMAINDER, FP8, U, WIDE, among_nans, as_type, check, check8, generator

pytestmark = pytest.mark.gpu
SIZES = [(1, 1), (1, 128), (3, 7), (5, 511), (4, 512), (7, 513), (9, 1000), (17, 1024), (33, 1512), (6, 2049), (40, 3328), (3, 4096), (2, 4097),
         (5, 8200), (3, 16384), (2, 16385), (3, 40000)]


def additions(cols):
    return 8 * (-(-cols // 512)) + 12


def forward(x, w, b, eps):
    """(m, r, n, y) and their errors."""
    cols = x.shape[1]
    m = x.mean(1, keepdim=True)
    em = additions(cols) * U * x.abs().mean(1, keepdim=True) + U * m.abs()
    d = x - m
    var = d.square().mean(1, keepdim=True) + eps
    r = 1 / var.sqrt()
    er = (em.square() / var + (additions(cols) + 6) * U) / 2 + 2 * U
    n = d * r
    en = n.abs() * (er + 3 * U) + em * r * (1 + er)
    ww, bb = (1.0 if w is None else w.double()), (0.0 if b is None else b.double())
    y = n * ww + bb
    ey = en * abs(ww) + 2 * U * ((n * ww).abs() + abs(bb))
    return (m, em + U * m.abs()), (r, er * r), (n, en), (y, ey)


def inputs(rows, cols, dtype, device, seed=0):
    g = generator(device, rows + cols + seed)
    x = torch.randn(rows, cols, generator=g, device=device) * torch.rand(rows, 1, generator=g, device=device).mul_(4).exp2_()
    x = (x + torch.randn(rows, 1, generator=g, device=device)).to(dtype)
    return x, torch.randn(cols, generator=g, device=device), torch.randn(cols, generator=g, device=device)


def check_forward(x, w, b, eps, out, **kw):
    got = train.layer_norm(x, w, b, eps, out_dtype=out, **kw)
    (m, em), (r, er), (n, en), (y, ey) = forward(x.double(), w, b, eps)
    if out == FP8:
        check8(got.y, got.y_scales, y, ey)
    else:
        check(got.y, y, ey, out)
    if got.mean is not None:
        check(got.mean[:, None], m, em, torch.float32)
    if got.rstd is not None:
        check(got.rstd[:, None], r, er, torch.float32)
    if got.kept is not None:
        check8(got.kept, got.kept_scales, n, en)
    return got


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", WIDE)
def test_forward(rows, cols, dtype, device):
    x, w, b = inputs(rows, cols, dtype, device)
    check_forward(x, w, b, 1e-5, torch.bfloat16, statistics=True)
    check_forward(x, w, None, 1e-5, FP8, checkpoint=True)
    check_forward(x, None, b, 1e-3, torch.float32)
    check_forward(x, None, None, 1e-5, torch.float16, checkpoint=True, statistics=True)


@pytest.mark.parametrize("cols", [189, 1512, 3328])
def test_forward_many_rows(cols, device):
    x, w, b = inputs(2500, cols, torch.float32, device)
    check_forward(x, w, b, 1e-5, torch.float16, checkpoint=True)
    check_forward(x, w, b, 1e-5, FP8, statistics=True)


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("rows,cols", [(2048, 8), (2051, 512), (2050, 520), (4099, 200), (2049, 1512), (2055, 2048), (2100, 2568), (2101, 3080), (2500, 4096)])
def test_forward_weights_held(rows, cols, dtype, device):
    """Rows that share their weights by eight; the last ones fewer."""
    x, w, b = inputs(rows, cols, dtype, device)
    check_forward(x, w, b, 1e-5, dtype, checkpoint=True)
    check_forward(x, w, None, 1e-5, FP8, statistics=True)
    check_forward(x, None, b, 1e-5, torch.bfloat16)


@pytest.mark.parametrize("dtype", WIDE)
def test_forward_strided(dtype, device):
    x, w, b = inputs(40, 900, dtype, device)
    for view in (x[3:, 5:777], x[::3, 1:130], x[1:2, 7:]):
        n = view.shape[1]
        check_forward(view, w[:n].contiguous(), b[:n].contiguous(), 1e-5, dtype, checkpoint=True)


def test_forward_special_rows(device):
    x = torch.zeros(8, 300, device=device)
    x[1] = 7.0                                   # constant: n = 0
    x[2, 5] = float("inf")
    x[3, 299] = float("nan")
    x[4] = torch.arange(300, device=device) % 2  # +-1 exactly
    x[5] = 1e-30 * torch.arange(300, device=device)
    x[6] = 1e4 + torch.arange(300, device=device)
    w, b = torch.full((300,), 2.0, device=device), torch.full((300,), -1.0, device=device)
    for out in (torch.float32, FP8):
        r = train.layer_norm(x, w, b, 1e-5, out_dtype=out, checkpoint=True, statistics=True)
        y = r.y.float()
        assert y[2:4].isnan().all() and r.kept[2:4].float().isnan().all() and not y[[0, 1, 4, 5, 6, 7]].isnan().any()
        for row in (0, 1, 7):
            assert (r.kept[row].float() == 0).all() and (r.kept_scales[row] == 2.0 ** -126).all()
        keep = [0, 1, 4, 5, 6, 7]
        check_forward(x[keep], w, b, 1e-5, out, checkpoint=True)
    zero = train.layer_norm(x[:2], eps=0.0, out_dtype=torch.float32, statistics=True)
    assert zero.rstd.isinf().all() and zero.y.isnan().all()  # 0 * infinity, as the formula has it


def test_no_rows(device):
    r = train.layer_norm(torch.empty(0, 70, device=device), out_dtype=FP8, checkpoint=True)
    assert r.y.shape == (0, 70) and r.kept_scales.shape == (0, 1)
    dx, dw, db = train.layer_norm_backward(torch.empty(0, 70, device=device), r.kept, r.rstd, x_scales=r.kept_scales)
    assert dx.shape == (0, 70) and (dw == 0).all() and (db == 0).all()


def test_row_offsets_past_32_bits(device):
    big = torch.empty(5, 1 << 29, dtype=torch.bfloat16, device=device)
    big[:, :300] = torch.randn(5, 300, generator=generator(device, 1), device=device).to(torch.bfloat16)
    check_forward(big[:, :300], None, None, 1e-5, torch.float32, statistics=True)


# ------------------------------------------------------------------------------- gradients


def backward(dy, n, r, w, en):
    """(dx, dweight, dbias) and their errors; n errs by en times itself."""
    rows, cols = dy.shape
    h, down = additions(cols) + 1, min(rows, rows / 512 + 140) + 4
    g = dy if w is None else dy * w.double()
    c1, c2 = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    e1 = (h + 2) * U * g.abs().mean(1, keepdim=True)
    e2 = ((h + 4) * U + en) * (g * n).abs().mean(1, keepdim=True)
    dx = r * (g - c1 - n * c2)
    ex_ = r * (4 * U * (g.abs() + c1.abs()) + e1 + n.abs() * e2 + (n * c2).abs() * (4 * U + en)) + U * dx.abs()
    each = (dy * n).abs().sum(0)
    return (dx, ex_), ((dy * n).sum(0), (down * U + 2 * U + en) * each), (dy.sum(0), down * U * dy.abs().sum(0))


def check_backward(dy, x, x_scales, mean, rstd, w):
    dx, dw, db = train.layer_norm_backward(dy, x, rstd, mean=mean, x_scales=x_scales, weight=w)
    r = rstd.double()[:, None]
    if x_scales is not None:
        n, en = x.double() * x_scales.double().repeat_interleave(128, 1)[:, :x.shape[1]], U
    else:
        n, en = (x.double() - mean.double()[:, None]) * r, 3 * U
    want = backward(dy.double(), n, r, w, en)
    check(dx, *want[0], dy.dtype)
    check(dw[None], want[1][0][None], want[1][1], torch.float32)
    check(db[None], want[2][0][None], want[2][1], torch.float32)
    only, none, nothing = train.layer_norm_backward(dy, x, rstd, mean=mean, x_scales=x_scales, weight=w, parameters=False)
    assert torch.equal(only, dx) and none is None and nothing is None


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dy_type,x_type", [(torch.float32, torch.float32), (torch.bfloat16, FP8), (torch.float16, torch.bfloat16),
                                            (torch.float32, FP8), (torch.bfloat16, torch.float16)])
def test_backward(rows, cols, dy_type, x_type, device):
    x, w, _ = inputs(rows, cols, torch.float32 if x_type == FP8 else x_type, device)
    dy = (torch.randn(rows, cols, generator=generator(device, cols), device=device) * 0.1).to(dy_type)
    r = train.layer_norm(x, statistics=True, checkpoint=x_type == FP8)
    if x_type == FP8:
        check_backward(dy, r.kept, r.kept_scales, None, r.rstd, w)
    else:
        check_backward(dy, x, None, r.mean, r.rstd, w)
        check_backward(dy, x, None, r.mean, r.rstd, None)


@pytest.mark.parametrize("rows,cols", [(2047, 189), (5000, 64), (3000, 1512), (1500, 3328), (4500, 700), (700, 8192)])
def test_backward_many_rows(rows, cols, device):
    x, w, _ = inputs(rows, cols, torch.float32, device)
    dy = (torch.randn(rows, cols, generator=generator(device, cols), device=device) * 0.1).to(torch.bfloat16)
    r = train.layer_norm(x, statistics=True, checkpoint=True)
    check_backward(dy, r.kept, r.kept_scales, None, r.rstd, w)
    check_backward(dy, x, None, r.mean, r.rstd, w)


def test_backward_strided(device):
    x, w, _ = inputs(50, 900, torch.float16, device)
    dy = torch.randn(50, 901, generator=generator(device, 5), device=device).to(torch.float16)
    r = train.layer_norm(x[::2, 3:700], statistics=True)
    check_backward(dy[::2, 2:699], x[::2, 3:700], None, r.mean, r.rstd, w[:697].contiguous())


def test_backward_is_the_slope(device):
    """Against differences of the definition, in 64 bits: (f(x + t v) - f(x - t v)) / 2 t = dx . v to t^2."""
    x, w, b = inputs(6, 200, torch.float32, device)
    dy = torch.randn(6, 200, generator=generator(device, 3), device=device)
    v = torch.randn(6, 200, generator=generator(device, 4), device=device).double()
    f = lambda x: torch.nn.functional.layer_norm(x, (200,), w.double(), b.double(), 1e-5)  # noqa: E731
    r = train.layer_norm(x, w, b, statistics=True)
    dx, dw, db = train.layer_norm_backward(dy, x, r.rstd, mean=r.mean, weight=w)
    t = 1e-5
    slope = ((f(x.double() + t * v) - f(x.double() - t * v)) / (2 * t) * dy.double()).sum()
    # fp32 statistics and sums: some hundred roundings; t^2 and 2^-53 / t are below.
    assert abs(slope - (dx.double() * v).sum()) <= 300 * U * (dx.double() * v).abs().sum() + 1e-6 * abs(slope)
    n = f(x.double()).sub(b.double()).div(w.double())
    assert ((dw.double() - (dy.double() * n).sum(0)).abs() <= 300 * U * (dy.double() * n).abs().sum(0) + 1e-9).all()


def test_graph_and_streams(device):
    """Two captured graphs with outputs and workspaces of their own, replayed between eager work, equal eager calls."""
    x, w, b = inputs(300, 1000, torch.float32, device)
    dy = torch.randn(300, 1000, generator=generator(device, 9), device=device).to(torch.bfloat16)

    def step():
        r = train.layer_norm(x, w, b, out_dtype=FP8, checkpoint=True)
        return (*r[:2], *r[3:], *train.layer_norm_backward(dy, r.kept, r.rstd, x_scales=r.kept_scales, weight=w))
    side = torch.cuda.Stream(device)
    side.wait_stream(torch.cuda.current_stream(device))
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append(step())
    for replay in range(3):
        x.copy_(torch.randn(300, 1000, generator=generator(device, 20 + replay), device=device))
        for o in outs:
            for t in o:
                t.view(torch.uint8 if t.dtype == FP8 else t.dtype).fill_(1)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for want, *got in zip(step(), *outs):
            for t in got:
                assert torch.equal(t.float(), want.float()), replay
    other = torch.cuda.Stream(device)
    other.wait_stream(torch.cuda.current_stream(device))
    y = train.layer_norm(x, w, b, stream=other).y
    torch.cuda.synchronize()
    assert torch.equal(y, train.layer_norm(x, w, b).y)


def test_refusals(device):
    x = torch.zeros(4, 32, device=device)
    r = train.layer_norm(x, statistics=True, checkpoint=True)
    w = torch.ones(32, device=device)
    for bad in (lambda: train.layer_norm(x.double()), lambda: train.layer_norm(x.cpu()), lambda: train.layer_norm(x.t()), lambda: train.layer_norm(x[0]),
                lambda: train.layer_norm(r.kept), lambda: train.layer_norm(x, w[:31]), lambda: train.layer_norm(x, w.double()),
                lambda: train.layer_norm(x, w, w.cpu()), lambda: train.layer_norm(x, out_dtype=torch.float64),
                lambda: train.layer_norm_backward(x, r.kept, r.rstd), lambda: train.layer_norm_backward(x, x, r.rstd),
                lambda: train.layer_norm_backward(x, r.kept, r.rstd, mean=r.mean, x_scales=r.kept_scales),
                lambda: train.layer_norm_backward(x, x, r.rstd, mean=r.mean, x_scales=r.kept_scales),
                lambda: train.layer_norm_backward(x, x[:3], r.rstd, mean=r.mean), lambda: train.layer_norm_backward(x, x, r.rstd[:3], mean=r.mean),
                lambda: train.layer_norm_backward(x, x.cpu(), r.rstd, mean=r.mean), lambda: train.layer_norm_backward(r.kept, x, r.rstd, mean=r.mean)):
        with pytest.raises(ValueError):
            bad()
    for eps in (-1.0, float("nan")):
        with pytest.raises(eb.EbError) as e:
            train.layer_norm(x, eps=eps)
        assert e.value.code == eb.EB_ERR_INVALID


@pytest.mark.parametrize("cols", EVERY_REMAINDER)
@pytest.mark.parametrize("dtype", WIDE)
def test_every_remainder(cols, dtype, device):
    """Rows that end anywhere in a chunk of 8, with NaN before and behind them."""
    x, w, b = inputs(19, cols, dtype, device)
    x = among_nans(x)
    dy = among_nans((torch.randn(19, cols, generator=generator(device, cols), device=device) * 0.1).to(dtype))
    r = check_forward(x, w, b, 1e-5, FP8, statistics=True, checkpoint=True)
    check_backward(dy, r.kept, r.kept_scales, None, r.rstd, w)
    check_backward(dy, x, None, r.mean, r.rstd, w)
