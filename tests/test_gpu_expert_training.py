"""The operators that train a layer of experts, run together (``ExpertTraining``), on pooled lookups.

The layer holds values in 8 bits, so each step is checked in 64 bits against what the step
before it left, within that step's own roundings (u = 2^-24): products of 8-bit rows are
exact to fp32's rounding or, for 16-bit outputs, within 1.5e-5 of the sum of their sizes and
2^-8; joined rows as in the tests of combine; weight gradients 2^-20 and the additions.
The whole is checked against differences of the layer in 64 bits, without 8-bit roundings:
there each of the five values in 8 bits is off by up to 2^-4 of itself (rms 2^-5.3), those
errors are independent, and an inner product of a gradient with a random direction averages
them: a tenth of the product of both norms is forty times what is left.
"""
import importlib.util
import os

import pytest
import torch

from paper_2512_05831_amd import experts as ex, train
from train_util import FP8, U, check, generator, held

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GATE, RELU = ex.EB_ACT_SILU_GATE, ex.EB_ACT_RELU


def layer_of(E, K, hidden, D, top, device, act=GATE, norm=True, experts=None, **kw):
    g = generator(device, E + K)
    N = 2 * hidden if act == GATE else hidden
    w_up = torch.randn(E, N, K, generator=g, device=device) * K ** -0.5
    w_down = torch.randn(E, D, hidden, generator=g, device=device) * hidden ** -0.5
    router = torch.randn(experts or E, K, generator=g, device=device) * K ** -0.5
    if norm:
        kw.update(norm_weight=1 + 0.1 * torch.randn(K, generator=g, device=device), norm_bias=0.1 * torch.randn(K, generator=g, device=device))
    return train.ExpertTraining(w_up, w_down, router, top, act, **kw)


def weights_held(form):
    q, s = form
    return q.double() * s.double().repeat_interleave(128, 1)[:, :q.shape[1]].repeat_interleave(128, 2)[:, :, :q.shape[2]]


def grouped(rows, w, offsets):
    """Slots times their experts' weights [E, out, in], and the sums of the sizes."""
    y, size = (torch.zeros(rows.shape[0], w.shape[1], dtype=torch.float64, device=rows.device) for _ in range(2))
    for e, (a, b) in enumerate(zip(offsets, offsets[1:])):
        y[a:b], size[a:b] = rows[a:b] @ w[e].t(), rows[a:b].abs() @ w[e].abs().t()
    return y, size


@pytest.mark.parametrize("B", [1, 7, 300])
@pytest.mark.parametrize("E,K,hidden,D,top,act,norm,shards", [(8, 256, 128, 64, 2, GATE, True, 1), (5, 378, 200, 100, 3, RELU, True, 1),
                                                              (6, 512, 300, 256, 4, GATE, False, 2)])
def test_each_step(B, E, K, hidden, D, top, act, norm, shards, device):
    layer = layer_of(E, K, hidden, D, top, device, act, norm, experts=E * shards)
    g = generator(device, B)
    x, dout = torch.randn(B, K, generator=g, device=device) * 0.3, torch.randn(B, D, generator=g, device=device).to(torch.bfloat16) * 1e-2
    out, s = layer.forward(x)
    r = s.route
    offsets = r.offsets.tolist()
    used = offsets[-1]
    # forward: the joined rows
    ok = r.slots >= 0
    z = s.rows.double()
    pick = torch.where(ok[:, :, None], z[r.slots.clamp(min=0).long()], 0.0) * r.weights.double()[:, :, None]
    check(out, pick.sum(1), (top + 1) * U * pick.abs().sum(1), torch.float32)
    grads, mid = layer._backward(s, dout)
    dz, dv, h = (held(*mid[k])[:used] for k in ("dz", "dv", "h"))
    X = held(*s.x)
    # the products back
    for got, rows, form in ((mid["dh"], dz, layer._down_t), (mid["dslots"], dv, layer._up_t)):
        want, size = grouped(rows, weights_held(form), offsets)
        check(got[:used], want, 2.0 ** -15 * size, torch.bfloat16)
    # the weights' gradients
    tokens = r.tokens[:used].long()
    for got, a, b in ((grads.w_down, dz, h), (grads.w_up, dv, X[tokens])):
        for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
            size = a[lo:hi].abs().t() @ b[lo:hi].abs()
            check(got[e], a[lo:hi].t() @ b[lo:hi], (2.0 ** -20 + (hi - lo + 40) * U) * size + 2.0 ** -30 * size.max(), torch.float32)
    # the router's, by autograd of the definition in 64 bits
    scores = s.scores.double().requires_grad_()
    p = torch.softmax(scores, 1).gather(1, r.ids.clamp(min=0).long())
    w = p / p.sum(1, keepdim=True)
    (w * mid["dweights"].double()).sum().backward()
    off = (mid["dscores"].double() - scores.grad).abs()
    assert (off <= 64 * U * (mid["dweights"].double().abs().sum(1, keepdim=True) + scores.grad.abs())).all()
    ds = mid["dscores"].to(torch.bfloat16).double()
    check(grads.router, ds.t() @ X, (2.0 ** -20 + (B + 40) * U) * (ds.abs().t() @ X.abs()), torch.float32)
    # the input's
    back = torch.where(ok[:, :, None], mid["dslots"].double()[r.slots.clamp(min=0).long()], 0.0)
    dx, size = back.sum(1) + mid["dscores"].double() @ layer.router.double(), back.abs().sum(1) + mid["dscores"].double().abs() @ layer.router.double().abs()
    err = (E * shards + top + 4) * U * size
    if not norm:
        check(grads.x, dx, err, torch.float32)
        assert grads.norm_weight is None
        return
    n, rs, wt = held(*s.kept), s.rstd.double()[:, None], layer.norm_weight.double()
    err = err + (dx.abs() + err) * 2.0 ** -8  # in bf16
    gg, ge = dx * wt, err * wt.abs()
    want = rs * (gg - gg.mean(1, keepdim=True) - n * (gg * n).mean(1, keepdim=True))
    slack = rs * (ge + ge.mean(1, keepdim=True) + n.abs() * (ge * n.abs()).mean(1, keepdim=True)) + 64 * U * rs * (gg.abs() + gg.abs().mean(1, keepdim=True) * (1 + n.square()))
    check(grads.x, want, slack, torch.bfloat16)
    check(grads.norm_weight, (dx * n).sum(0), (err * n.abs()).sum(0) + (B + 8) * U * (dx * n).abs().sum(0), torch.float32)
    check(grads.norm_bias, dx.sum(0), err.sum(0) + (B + 8) * U * dx.abs().sum(0), torch.float32)


def exact_loss(layer, x, dout, ids, w_up, w_down, router, nw, nb):
    """The layer in 64 bits, its experts chosen as given."""
    y = torch.nn.functional.layer_norm(x, (layer.K,), nw, nb, layer.eps)
    p = torch.softmax(y @ router.t(), 1).gather(1, ids)
    w = p / p.sum(1, keepdim=True)
    out = 0
    for k in range(layer.top):
        v = torch.bmm(w_up[ids[:, k]], y[:, :, None])[:, :, 0]
        g, u = v.chunk(2, 1)
        h = g * torch.sigmoid(g) * u
        out = out + w[:, k, None] * torch.bmm(w_down[ids[:, k]], h[:, :, None])[:, :, 0]
    return (out * dout).sum()


def test_against_differences(device):
    layer = layer_of(8, 256, 128, 64, 2, device)
    g = generator(device, 1)
    x, dout = torch.randn(64, 256, generator=g, device=device), torch.randn(64, 64, generator=g, device=device)
    _, s = layer.forward(x)
    grads = layer.backward(s, dout)
    ids = s.route.ids.long()
    at = [t.double() for t in (x, layer.w_up, layer.w_down, layer.router, layer.norm_weight, layer.norm_bias)]
    f = lambda p: exact_loss(layer, p[0], dout.double(), ids, *p[1:])  # noqa: E731
    for i, grad in enumerate(grads):
        # along the gradient itself, where the inner product is its square
        d = grad.double()
        t = 1e-4 / float(d.norm())
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + t * d, at[i] - t * d
        slope = float(f(up) - f(down)) / (2 * t)
        assert abs(slope / float(d.square().sum()) - 1) < 0.1, (i, slope, float(d.square().sum()))


def test_graph(device):
    """A step captured into a graph and replayed, between eager ones, equals them."""
    layer = layer_of(8, 256, 128, 64, 2, device)
    x, dout = torch.randn(100, 256, generator=generator(device, 2), device=device), torch.randn(100, 64, generator=generator(device, 3), device=device)

    def step():
        out, s = layer.forward(x)
        return (out, *layer.backward(s, dout))
    side = torch.cuda.Stream(device)
    side.wait_stream(torch.cuda.current_stream(device))
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for replay in range(3):
        x.copy_(torch.randn(100, 256, generator=generator(device, 10 + replay), device=device))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b), replay


def test_refresh(device):
    layer = layer_of(4, 128, 128, 64, 2, device, norm=False)
    x = torch.randn(20, 128, generator=generator(device, 2), device=device)
    before = layer.forward(x)[0]
    layer.w_down *= 2
    assert torch.equal(layer.forward(x)[0], before)
    layer.refresh()
    assert torch.equal(layer.forward(x)[0], 2 * before)


def test_refresh_and_a_captured_graph(device):
    """A graph captured before weights changed reads their new forms; one that holds refresh makes them."""
    layer = layer_of(4, 200, 72, 64, 2, device)
    x = torch.randn(20, 200, generator=generator(device, 2), device=device)
    side = torch.cuda.Stream(device)
    side.wait_stream(torch.cuda.current_stream(device))
    with torch.cuda.stream(side):
        layer.forward(x)
        layer.refresh()
    torch.cuda.synchronize()
    graph, both = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, _ = layer.forward(x)
    with torch.cuda.graph(both, stream=side):
        layer.refresh()
        fresh, _ = layer.forward(x)
    for replay in range(3):
        layer.w_up += 0.01 * torch.randn(layer.w_up.shape, generator=generator(device, 5 + replay), device=device)
        layer.w_down *= 1.5
        layer.refresh()
        other = train.ExpertTraining(layer.w_up, layer.w_down, layer.router, 2, norm_weight=layer.norm_weight, norm_bias=layer.norm_bias)
        want = other.forward(x)[0]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.forward(x)[0], want) and torch.equal(out, want), replay
        layer.w_down *= 0.5
        want = train.ExpertTraining(layer.w_up, layer.w_down, layer.router, 2, norm_weight=layer.norm_weight,
                                    norm_bias=layer.norm_bias).forward(x)[0]
        torch.cuda.synchronize()
        both.replay()
        torch.cuda.synchronize()
        assert torch.equal(fresh, want), replay
    layer.w_up = layer.w_up[:, :, :128]
    with pytest.raises(ValueError):
        layer.refresh()


@pytest.mark.parametrize("norm", [False, True])
def test_weights_that_require_gradients(norm, device):
    """Torch records nothing: what is returned and kept holds no graph."""
    plain, layer = (layer_of(8, 256, 128, 64, 2, device, norm=norm) for _ in range(2))
    for w in (layer.w_up, layer.w_down, layer.router, *((layer.norm_weight, layer.norm_bias) if norm else ())):
        w.requires_grad_(True)
    x, dout = torch.randn(50, 256, generator=generator(device, 2), device=device), torch.randn(50, 64, generator=generator(device, 3), device=device)
    layer.refresh()
    out, s = layer.forward(x.clone().requires_grad_(True))
    grads = layer.backward(s, dout.clone().requires_grad_(True))
    want_out, want_s = plain.forward(x)
    for got, want in zip((out, s.scores, *s.x, *s.v, s.rows, *grads), (want_out, want_s.scores, *want_s.x, *want_s.v, want_s.rows,
                                                                     *plain.backward(want_s, dout))):
        assert (got is None and want is None) or (not got.requires_grad and torch.equal(got.float(), want.float()))


def test_no_tokens(device):
    layer = layer_of(4, 128, 128, 64, 2, device)
    out, s = layer.forward(torch.empty(0, 128, device=device))
    grads = layer.backward(s, torch.empty(0, 64, device=device))
    assert out.shape == (0, 64) and grads.x.shape == (0, 128)
    assert all((g == 0).all() for g in grads[1:])


def test_refusals(device):
    w_up, w_down, router = torch.zeros(4, 256, 128, device=device), torch.zeros(4, 64, 128, device=device), torch.zeros(4, 128, device=device)
    for bad in (lambda: train.ExpertTraining(w_up[0], w_down, router, 2), lambda: train.ExpertTraining(w_up, w_down, router[:, :100], 2),
                lambda: train.ExpertTraining(w_up, w_down, router, 2, act=RELU), lambda: train.ExpertTraining(w_up, w_down, router, 2, act=ex.EB_ACT_NONE),
                lambda: train.ExpertTraining(w_up, w_down, router, 2, norm_weight=router[0])):
        with pytest.raises(ValueError):
            bad()
    layer = train.ExpertTraining(w_up, w_down, router, 2)
    for bad in (torch.zeros(3, 100, device=device), torch.zeros(128, device=device), torch.zeros(3, 128)):
        with pytest.raises(ValueError):
            layer.forward(bad)


def test_example(device):
    """The example's step runs, and its gradients are what the layer gives."""
    spec = importlib.util.spec_from_file_location("example", os.path.join(ROOT, "examples", "train_experts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    et, layer = example.build(tables=2, rows=1000, dim=64, experts=4, hidden=128, out=32, top=2)
    ids, offsets, target = example.batch(et, 50, 5, 32)
    loss, grads = example.step(et, layer, ids, offsets, target, 50, rate=0.0)
    assert torch.isfinite(loss) and all(torch.isfinite(g).all() for g in grads)
    pooled = et.forward(ids, offsets, 50)
    out, s = layer.forward(pooled)
    again = layer.backward(s, (out - target) * (2 / out.numel()))
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
