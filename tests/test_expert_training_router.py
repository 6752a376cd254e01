"""The gradient of the router's outputs in ``train.ExpertTraining``, against autograd of the definition in 64 bits.

Weights are exponentials against the largest of the chosen (or of all) over their sum: each
errs by (|x - largest| + 8) u of itself, u = 2^-24, of which the first part is below 0.4 u of 1.  A
gradient is scale w (d - sum w d), times 1 - p under a sigmoid: within 40 u |scale| sum |d|.
"""
from types import SimpleNamespace

import pytest
import torch

from paper_2512_05831_amd import experts as ex, train

U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")
SOFT, SIG, RENORM = ex.EB_SOFTMAX, ex.EB_SIGMOID, ex.EB_RENORMALIZE
MODES = [SOFT | RENORM, SOFT, SIG | RENORM, SIG]


def weights_of(scores, ids, mode, scale):
    """The route's weights from scores in 64 bits; every row of ids names an expert or none (-1)."""
    there = ids >= 0
    x = scores.gather(1, ids.clamp(min=0).long())
    # ln of each weight before it is renormalised (which takes out what all have: of a softmax the sum over all experts)
    log = torch.nn.functional.logsigmoid(x) if mode & 0xFF == SIG else x if mode & RENORM else x - torch.logsumexp(scores, 1, keepdim=True)
    if mode & RENORM:
        log = torch.log_softmax(log.masked_fill(~there, -INF), 1)
    return scale * torch.where(there, log.exp(), 0.0)


def expected(scores, ids, d, mode, scale):
    s = scores.double().clone()
    s[s == INF] = torch.finfo(torch.float32).max
    s[s.isnan()] = -INF
    got = torch.zeros_like(s)
    for n in range(len(s)):  # a row without a choice has no gradient
        if (ids[n] >= 0).any():
            row = s[n:n + 1].clone().requires_grad_()
            (weights_of(row, ids[n:n + 1], mode, scale) * d[n:n + 1].double()).sum().backward()
            got[n] = row.grad[0].nan_to_num(0.0)
    return got


def check(scores, ids, d, mode, scale):
    layer = SimpleNamespace(mode=mode, scale=scale)
    saved = SimpleNamespace(scores=scores, route=SimpleNamespace(ids=ids))
    got = train.ExpertTraining._dscores(layer, saved, d)
    want = expected(scores, ids, d, mode, scale)
    assert got.dtype == torch.float32 and got.shape == want.shape
    bound = 40 * U * abs(scale) * d.double().abs().sum(1, keepdim=True) + 2.0 ** -120
    assert ((got.double() - want).abs() <= bound).all(), (got, want)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("scale", [1.0, 2.5, -0.5, 0.0])
def test_of_random_scores(mode, scale):
    g = torch.Generator().manual_seed(mode + 1)
    scores = 3 * torch.randn(50, 12, generator=g)
    ids = torch.rand(50, 12, generator=g).topk(4, 1).indices.int()  # any four: as a bias may choose them
    ids[3, 2:], ids[4] = -1, -1
    check(scores, ids, torch.randn(50, 4, generator=g), mode, scale)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("above", [0.0, 60.0, 85.0, 95.0, 104.0, 120.0, 200.0, 1e4, 1e30])
def test_an_expert_kept_out_far_above(mode, above):
    """By a bias or its group: the chosen ones' share of all is nothing, their weights are not."""
    scores = torch.tensor([[above, 0.0, 0.5, -1.0], [above, 0.0, 0.0, above]])
    ids = torch.tensor([[2, 1], [1, 2]], dtype=torch.int32)
    check(scores, ids, torch.tensor([[1.0, 0.0], [0.3, -2.0]]), mode, 1.0)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("low", [-20.0, -87.0, -100.0, -120.0, -1e4])
def test_scores_far_below_zero(mode, low):
    scores = torch.tensor([[low, low + 0.5, low - 1.0, 2 * low]])
    for ids in ([[1, 0]], [[1, 3]], [[1, -1]]):
        check(scores, torch.tensor(ids, dtype=torch.int32), torch.tensor([[1.0, -0.5]]), mode, 1.5)


@pytest.mark.parametrize("mode", MODES)
def test_infinite_scores_and_nan(mode):
    """As the route takes them: an infinity as the largest float, minus infinity and NaN as experts that cannot be chosen."""
    scores = torch.tensor([[INF, 1.0, 0.0, -INF], [NAN, 1.0, 0.5, 0.0], [-INF, NAN, -INF, NAN], [1.0, -INF, NAN, 0.25]])
    ids = torch.tensor([[0, 1], [1, 2], [-1, -1], [0, 3]], dtype=torch.int32)
    check(scores, ids, torch.tensor([[1.0, -0.5], [0.25, 2.0], [1.0, 1.0], [1.0, 3.0]]), mode, 1.0)
