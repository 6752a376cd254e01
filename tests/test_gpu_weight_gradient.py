"""GPU parity of eb_weight_gradient with its definition in 64 bits.

A sum of c products passes fewer than c + 40 additions: (c + 40) u of the sum of their
sizes (u = 2^-24).  The products are within 2^-20 (fp32 and fp16 outputs), or 2^-8 (one
rounding to bfloat16), and where the scaled operand is in fp16 within 2^-34 of 448^2
times the largest product of a slot's two scales.
"""
import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex, train
from train_util import FP8, U, as_type, check, generator, route_of

pytestmark = pytest.mark.gpu
HALF, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = [(BF16, FP8), (FP8, FP8), (BF16, BF16), (HALF, HALF), (HALF, FP8), (FP8, HALF), (FP8, BF16), (HALF, BF16), (BF16, HALF)]


def operands(M, rows, N, K, dy_type, x_type, device, seed=0):
    g = generator(device, M + N + K + seed)
    sized = lambda r, c: torch.randn(r, c, generator=g, device=device) * torch.rand(r, 1, generator=g, device=device).add_(0.05)  # noqa: E731
    return as_type(sized(M, N) * 1e-2, dy_type), as_type(sized(rows, K), x_type)


def expected(dy, x, bounds, tokens, out, types):
    """[E, N, K] and its error."""
    (_, ds, dv), (_, xs, xv) = dy, x
    E, (M, N), K = len(bounds) - 1, dv.shape, xv.shape[1]
    want, err = torch.zeros(E, N, K, dtype=torch.float64, device=dv.device), torch.zeros(E, N, K, dtype=torch.float64, device=dv.device)
    half = BF16 not in types and FP8 in types
    for e in range(E):
        a, b = min(max(bounds[e], 0), M), min(max(bounds[e + 1], 0), M)
        if b <= a:
            continue
        m = torch.arange(a, b, device=dv.device)
        at = m if tokens is None else tokens[a:b].long()
        ok = (at >= 0) & (at < xv.shape[0])
        m, at = m[ok], at[ok]
        d, v = dv[m], xv[at]
        want[e] = d.t() @ v
        each = 2.0 ** -8 if out == BF16 else 2.0 ** -20
        err[e] = (each + (b - a + 40) * U) * (d.abs().t() @ v.abs())
        if half and len(m):
            s = torch.ones(len(m), 1, dtype=torch.float64, device=dv.device)
            largest = lambda t, v: (448 * t.double()).amax(1, keepdim=True) if t is not None else torch.ones_like(v[:, :1])  # noqa: E731
            scaled = largest(ds[m] if ds is not None else None, d) * largest(xs[at] if xs is not None else None, v)
            other = 1.0 if None not in (ds, xs) else (d if ds is None else v).abs().amax()
            err[e] += 2.0 ** -34 * float(scaled.max()) * other * len(m)
    return want, err


def run(M, E, N, K, types, out, device, rows=None, bounds=None, tokens=None, seed=0, **kw):
    dy, x = operands(M, M if rows is None else rows, N, K, *types, device, seed)
    offsets = None if bounds is None else torch.tensor(bounds, dtype=torch.int32, device=device)
    got = train.weight_gradient(dy[0], x[0], offsets=offsets, tokens=tokens, dy_scales=dy[1], x_scales=x[1], out_dtype=out, **kw)
    want, err = expected(dy, x, [0, M] if bounds is None else bounds, tokens, out, types)
    check(got if bounds is not None else got[None], want, err, out)
    return dy, x, got, want, err


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("out", [F32, BF16, HALF])
def test_types(types, out, device):
    run(200, 1, 150, 140, types, out, device)
    run(3, 1, 128, 256, types, out, device)
    run(700, 3, 70, 300, types, out, device, bounds=[0, 400, 401, 700])


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 5, 3), (63, 127, 129), (64, 128, 128), (65, 129, 127), (129, 1, 400), (130, 300, 2), (1000, 257, 131),
                                   (2048, 1000, 1512), (5000, 100, 60), (20000, 33, 65)])
@pytest.mark.parametrize("types", [(BF16, FP8), (FP8, FP8), (HALF, HALF)])
def test_one_expert(M, N, K, types, device):
    run(M, 1, N, K, types, F32, device)


@pytest.mark.parametrize("types", [(BF16, FP8), (FP8, FP8), (BF16, BF16)])
@pytest.mark.parametrize("N_tokens,E,top,shards", [(1, 8, 2, 1), (50, 8, 3, 1), (300, 40, 4, 1), (2000, 5, 2, 2)])
def test_routed(N_tokens, E, top, shards, types, device):
    """From tokens where they stand; experts without slots give zeros; pairs of other GPUs add nothing."""
    r = route_of(N_tokens, E, top, device, E, shards)
    run(N_tokens * top, len(r.offsets) - 1, 200, 136, types, F32, device, rows=N_tokens, bounds=r.offsets.tolist(), tokens=r.tokens)


def test_empty(device):
    dy, x, got, _, _ = run(10, 4, 9, 40, (BF16, FP8), F32, device, bounds=[0, 0, 10, 10, 10])
    assert (got[[0, 2, 3]] == 0).all()
    for out in (F32, HALF):
        z = train.weight_gradient(torch.empty(0, 9, device=device).half(), torch.empty(0, 40, device=device).half(), out_dtype=out)
        assert z.shape == (9, 40) and (z == 0).all()


def test_odd_offsets_and_tokens(device):
    """Offsets past the slots, negative or falling; tokens out of range: what lies there adds nothing, NaNs too."""
    M = 300
    tokens = torch.randint(-2, 52, (M,), generator=generator(device, 1), device=device, dtype=torch.int64).int()
    tokens[7], tokens[100] = -2147483648, 2147483647
    run(M, 4, 60, 50, (FP8, FP8), F32, device, rows=50, bounds=[-5, 100, 90, 400, 500], tokens=tokens)
    dy, x = operands(M, 50, 60, 50, BF16, BF16, device)
    dy[0][(tokens < 0) | (tokens >= 50)] = float("nan")
    got = train.weight_gradient(dy[0], x[0], tokens=tokens)
    dv = torch.where(dy[0].isnan(), 0.0, dy[0].double())
    check(got[None], *expected((dy[0], None, dv), x, [0, M], tokens, F32, (BF16, BF16)), F32)


@pytest.mark.parametrize("out", [F32, BF16, HALF])
@pytest.mark.parametrize("M,E", [(4000, 1), (100, 3)])
def test_accumulate_and_strides(M, E, out, device):
    """Added to what is there, rows of dw further apart; what lies between them stays."""
    bounds = None if E == 1 else [0, 30, 30, 100]
    dy, x, _, want, err = run(M, E, 40, 50, (BF16, FP8), out, device, bounds=bounds)
    room = torch.randn(E, 40, 61, generator=generator(device, 2), device=device).to(out)
    before = room.clone()
    dw = room[:, :, 3:53] if E > 1 else room[0, :, 3:53]
    offsets = None if E == 1 else torch.tensor(bounds, dtype=torch.int32, device=device)
    got = train.weight_gradient(dy[0], x[0], offsets=offsets, dy_scales=dy[1], x_scales=x[1], out=dw, accumulate=True)
    assert got.data_ptr() == dw.data_ptr()
    old = before[:, :, 3:53].double()
    check(room[:, :, 3:53], old + want, err + U * (old.abs() + want.abs()), out)
    assert torch.equal(room[:, :, :3], before[:, :, :3]) and torch.equal(room[:, :, 53:], before[:, :, 53:])
    train.weight_gradient(dy[0], x[0], offsets=offsets, dy_scales=dy[1], x_scales=x[1], out=dw)
    check(room[:, :, 3:53], want, err, out)


@pytest.mark.parametrize("types", [(BF16, BF16), (HALF, HALF)])
def test_strided_operands(types, device):
    g = generator(device, 3)
    dy, x = torch.randn(333, 210, generator=g, device=device).to(types[0]), torch.randn(333, 190, generator=g, device=device).to(types[1])
    for a, b in ((dy[:, 3:200], x[:, 1:140]), (dy[::3, :77], x[::3, 5:6]), (dy[5:6], x[7:8])):
        got = train.weight_gradient(a, b)
        want = a.double().t() @ b.double()
        check(got, want, (2.0 ** -20 + (len(a) + 40) * U) * (a.double().abs().t() @ b.double().abs()), F32)


def test_scales_that_grow_and_shrink(device):
    """Slots whose scales differ by 2^60, growing, falling and mixed: the large ones keep their precision, and slots
    of small scales theirs among themselves."""
    g = generator(device, 4)
    for M, power in ((512, torch.arange(512) * 60 // 512), (512, 60 - torch.arange(512) * 60 // 512), (900, torch.randint(0, 60, (900,)))):
        size = torch.exp2(power.to(device).float() - 40)[:, None]
        dy = as_type(torch.randn(M, 130, generator=g, device=device) * size, FP8)
        x = as_type(torch.randn(M, 140, generator=g, device=device), FP8)
        for out in (F32, BF16):
            got = train.weight_gradient(dy[0], x[0], dy_scales=dy[1], x_scales=x[1], out_dtype=out)
            want, err = expected(dy, x, [0, M], None, out, (FP8, FP8))
            check(got[None], want, err, out)
    small = as_type(torch.randn(70, 130, generator=g, device=device) * 1e-36, FP8)
    x = as_type(torch.randn(70, 140, generator=g, device=device), FP8)
    got = train.weight_gradient(small[0], x[0], dy_scales=small[1], x_scales=x[1])
    want, err = expected(small, x, [0, 70], None, F32, (FP8, FP8))
    check(got[None], want, err + 2.0 ** -126, F32)


def test_rms_error_of_exact_sums(device):
    """Sums of 1000 products in fp32: a random walk of roundings is about sqrt(1000) / 2 * u of the result's size; 2e-6 is twice that."""
    for types in ((FP8, FP8), (BF16, FP8), (FP8, HALF), (HALF, BF16), (BF16, BF16)):
        dy, x = operands(1000, 1000, 256, 256, *types, device)
        got = train.weight_gradient(dy[0], x[0], dy_scales=dy[1], x_scales=x[1]).double()
        want = dy[2].t() @ x[2]
        assert float((got - want).norm() / want.norm()) < 2e-6, types


def test_nan_and_infinity_stay_in_their_rows(device):
    dy, x = operands(100, 100, 130, 130, BF16, BF16, device)
    dy[0][5, 7], x[0][9, 3] = float("inf"), float("nan")
    got = train.weight_gradient(dy[0], x[0])
    bad = torch.zeros(130, 130, dtype=torch.bool, device=device)
    bad[7], bad[:, 3] = True, True
    assert torch.equal(~got.isfinite(), bad)


def test_against_differences(device):
    """The product is linear in the weights: its change along dW is the gradient's inner product with that."""
    g = generator(device, 6)
    r = route_of(60, 4, 2, device, 6)
    x, up = torch.randn(60, 64, generator=g, device=device).to(BF16), torch.randn(120, 48, generator=g, device=device).to(BF16)
    dw = train.weight_gradient(up, x, offsets=r.offsets, tokens=r.tokens).double()
    W, V = (torch.randn(4, 48, 64, generator=g, device=device).double() for _ in range(2))
    of = torch.repeat_interleave(torch.arange(4, device=device), r.offsets.diff().long())
    f = lambda W: ((W[of] @ x.double()[r.tokens.long()][:, :, None])[:, :, 0] * up.double()).sum()  # noqa: E731
    t = 1e-3
    slope = (f(W + t * V) - f(W - t * V)) / (2 * t)
    assert abs(slope - (dw * V).sum()) <= 1e-5 * (dw * V).abs().sum()


def test_graph_and_streams(device):
    """Two captured graphs with workspaces of their own, replayed between eager work; another stream."""
    dy, x = operands(3000, 3000, 100, 200, BF16, FP8, device)
    call = lambda **kw: train.weight_gradient(dy[0], x[0], dy_scales=dy[1], x_scales=x[1], **kw)  # noqa: E731
    assert train.eb_weight_gradient_workspace(3000, 1, 100, 200) > 0
    side = torch.cuda.Stream(device)
    side.wait_stream(torch.cuda.current_stream(device))
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph in graphs:
        with torch.cuda.graph(graph, stream=side):
            outs.append(call())
    for replay in range(3):
        dy[0].copy_(torch.randn(3000, 100, generator=generator(device, replay), device=device))
        for o in outs:
            o.fill_(9)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = call()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    other = torch.cuda.Stream(device)
    other.wait_stream(torch.cuda.current_stream(device))
    got = call(stream=other)
    torch.cuda.synchronize()
    assert torch.equal(got, call())


def test_refusals(device):
    d, x = torch.zeros(4, 32, device=device).half(), torch.zeros(4, 16, device=device).half()
    q, s = ex.quantize_fp8(x)
    i, off = torch.zeros(4, dtype=torch.int32, device=device), torch.tensor([0, 2, 4], dtype=torch.int32, device=device)
    f = train.weight_gradient
    for bad in (lambda: f(d, q), lambda: f(d, x, x_scales=s), lambda: f(d[0], x), lambda: f(d.t(), x), lambda: f(d, x.cpu()), lambda: f(d.cpu(), x),
                lambda: f(d, x, offsets=off.long()), lambda: f(d, x, offsets=off[:1]), lambda: f(d, x, tokens=i[:3]), lambda: f(d, x, tokens=i.cpu()),
                lambda: f(d, x, accumulate=True), lambda: f(d, x, out=torch.zeros(32, 15, device=device)),
                lambda: f(d, x, offsets=off, out=torch.zeros(32, 16, device=device)), lambda: f(d, x, out_dtype=F32, out=torch.zeros(32, 16, device=device).half()),
                lambda: f(d, x, out=torch.zeros(32, 16)), lambda: f(d, x, out_dtype=FP8), lambda: f(d, q, x_scales=s.half()),
                lambda: f(d, x, offsets=off, out=torch.zeros(4, 32, 16, device=device)[::2])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(d.float(), x), lambda: f(d, x.float()), lambda: f(d, x[:3])):
        with pytest.raises(eb.EbError) as e:
            bad()
        assert e.value.code == eb.EB_ERR_INVALID
