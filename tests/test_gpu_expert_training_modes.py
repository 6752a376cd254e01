"""``ExpertTraining`` under every mode of the router: the gradients that pass through it, against the definition in 64 bits
(bounds as in test_expert_training_router.py), and the shares of several GPUs against one GPU's whole."""
import pytest
import torch

from paper_2512_05831_amd import experts as ex, train
from train_util import generator
from test_expert_training_router import INF, MODES, RENORM, SIG, U, expected, weights_of
from test_gpu_expert_training import GATE, layer_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("scale", [1.0, 2.5])
@pytest.mark.parametrize("kept_out", ["none", "by bias", "by group"])
@pytest.mark.parametrize("shard_lo,held", [(0, 8), (4, 4)])
def test_modes(mode, scale, kept_out, shard_lo, held, device):
    kw = {}
    if kept_out == "by bias":
        kw["bias"] = torch.tensor([-INF, 0.0, 5.0, 0.0, -INF, 0.1, 0.0, 0.0], device=device)
    elif kept_out == "by group":
        kw.update(groups=4, top_groups=2, mode=mode | ex.EB_GROUP_PAIR)
    layer = layer_of(held, 128, 64, 32, 3, device, norm=False, experts=8, scale=scale, shard_lo=shard_lo, **{"mode": mode, **kw})
    g = generator(device, 5)
    x, dout = torch.randn(40, 128, generator=g, device=device), torch.randn(40, 32, generator=g, device=device)
    if kept_out == "by bias":
        x[:7] = 250 * layer.router[0]  # the expert that is kept out lies far above
    out, s = layer.forward(x)
    ids = s.route.ids
    want_w = weights_of(s.scores.double(), ids, mode, scale)
    assert ((s.route.weights.double() - want_w).abs() <= 64 * U * scale).all()
    grads, mid = layer._backward(s, dout)
    d = mid["dweights"]
    assert (d[s.route.slots < 0] == 0).all()
    want = expected(s.scores, ids, d, mode, scale)
    assert ((mid["dscores"].double() - want).abs() <= 40 * U * scale * d.double().abs().sum(1, keepdim=True) + 2.0 ** -120).all()
    assert all(bool(t.isfinite().all()) for t in (grads.x, grads.w_up, grads.w_down, grads.router))


def test_shares_add_up(device):
    """Two GPUs' gradients of x and the router add up to one GPU's.  The same slots' rows: what differs is the order of fp32
    sums, and bf16 roundings of rows by products of other sizes (2^-8 of each)."""
    g = generator(device, 6)
    x, dout = torch.randn(64, 128, generator=g, device=device), torch.randn(64, 32, generator=g, device=device)
    whole = layer_of(8, 128, 64, 32, 3, device, norm=False, mode=SIG | RENORM, scale=1.5)
    out, s = whole.forward(x)
    want = whole.backward(s, dout)
    parts = []
    for lo in (0, 4):
        part = train.ExpertTraining(whole.w_up[lo:lo + 4], whole.w_down[lo:lo + 4], whole.router, 3, GATE, SIG | RENORM, scale=1.5, shard_lo=lo)
        y, saved = part.forward(x)
        parts.append((y, part.backward(saved, dout)))
    near = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm()) < 2.0 ** -7  # noqa: E731
    assert near(parts[0][0] + parts[1][0], out)
    assert near(parts[0][1].x + parts[1][1].x, want.x) and near(parts[0][1].router + parts[1][1].router, want.router)
    for lo, (_, grads) in zip((0, 4), parts):
        assert near(grads.w_up, want.w_up[lo:lo + 4]) and near(grads.w_down, want.w_down[lo:lo + 4])
