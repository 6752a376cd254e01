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
