"""Weights and groups of eb_route_experts in every kernel: with and without
renormalising, with a bias, groups and pairs, for few tokens (one workgroup) and
many, against the plain implementation in 64 bits and under its bounds.
"""
import pytest
import torch

from paper_2512_05831_amd import experts as ex
from test_gpu_route_experts import INF, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [INF, -INF, float("nan"), 0.0, -1.5])
@pytest.mark.parametrize("N", [3, 200, 3000])
def test_a_pair_without_an_expert_weighs_nothing(N, scale, device):
    """0 where the id is -1, whatever the scale."""
    x = torch.randn(N, 64, generator=torch.Generator().manual_seed(N), dtype=torch.float32)
    x[::3, 2:] = -INF
    for mode in (ex.EB_SOFTMAX, ex.EB_SIGMOID, ex.EB_SOFTMAX | ex.EB_RENORMALIZE, ex.EB_SIGMOID | ex.EB_RENORMALIZE):
        r = ex.route(x.to(device), 6, mode=mode, scale=scale)
        assert (r.ids[::3, 2:] == -1).all() and (r.ids[1::3] >= 0).all()
        assert (r.weights[r.ids < 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("function", [ex.EB_SOFTMAX, ex.EB_SIGMOID])
@pytest.mark.parametrize("E,K,groups,top_groups", [(40, 3, 5, 2), (64, 6, 8, 3), (100, 6, 10, 3), (160, 6, 8, 3), (256, 8, 8, 4), (510, 20, 17, 6)])
@pytest.mark.parametrize("judge", ["best", "pair", "bias", "bias+pair"])
@pytest.mark.parametrize("N", [1, 5, 16, 203])
def test_groups_with_and_without_renormalising(dtype, function, E, K, groups, top_groups, judge, N, device):
    g = torch.Generator().manual_seed(E + K + N)
    x = torch.randn(N, E, generator=g).to(dtype)
    bias = 0.1 * torch.randn(E, generator=g) if "bias" in judge else None
    mode = function | (ex.EB_GROUP_PAIR if "pair" in judge else 0)
    for renormalize in (0, ex.EB_RENORMALIZE):
        check(x, K, device, mode | renormalize, bias, groups, top_groups, 2.5, lo=E // 4, hi=E // 2, least_clear=0.5)


@pytest.mark.parametrize("function", [ex.EB_SOFTMAX, ex.EB_SIGMOID])
@pytest.mark.parametrize("N,E,K", [(1, 20, 4), (16, 64, 5), (100, 64, 8), (16, 128, 3), (16, 300, 9), (700, 32, 2), (700, 96, 7), (700, 200, 20), (300, 1000, 8)])
def test_biased_choice_without_renormalising(function, N, E, K, device):
    """The weights are the scores themselves: no bias in them, all experts in the softmax's sum."""
    g = torch.Generator().manual_seed(N + E)
    x = 2 * torch.randn(N, E, generator=g)
    x[:, 1] = -INF
    check(x, K, device, function, torch.linspace(-1, 1, E)[torch.randperm(E, generator=g)], scale=0.5, least_clear=0.5)


@pytest.mark.parametrize("N", [2, 300])
def test_weights_under_a_bias_with_nan_and_infinity(N, device):
    x = torch.zeros(N, 20)
    bias = torch.linspace(-1, 1, 20)
    bias[19], bias[18], bias[17] = float("nan"), INF, -INF
    for function, s in ((ex.EB_SIGMOID, 0.5), (ex.EB_SOFTMAX, 1 / 20)):
        r = ex.route(x.to(device), 20, mode=function, bias=bias.to(device))
        assert (r.ids == torch.tensor([18] + list(range(16, -1, -1)) + [-1, -1], dtype=torch.int32, device=device)).all()
        assert ((r.weights[:, :18].double() - s).abs() <= 36 * 2.0 ** -24 * s).all() and (r.weights[:, 18:] == 0).all()
        r = ex.route(x.to(device), 20, mode=function | ex.EB_RENORMALIZE, bias=bias.to(device))
        assert ((r.weights[:, :18].double() - 1 / 18).abs() <= 36 * 2.0 ** -24 / 18).all() and (r.weights[:, 18:] == 0).all()
