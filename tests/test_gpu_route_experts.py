"""GPU parity of eb_route_experts with a plain implementation in 64 bits.

Whole numbers are compared exactly.  Where the choice rests on rounded scores
(a bias, or pairs judging a group), a token whose decisions have a margin below
the scores' rounding is left out: s has at most 4 rounding errors of 2^-24 of a
value up to 1 (the exponential's, the sum's or 1 + e, the division's), the bias
and the pair add one each, so margins above MARGIN decide the same way.
Weights: a softmax adds E exponentials in fp32, so |w - exact| <= (E + 16) 2^-24 |w|, and
2^-126 where a weight leaves fp32's range.
"""
import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex

pytestmark = pytest.mark.gpu
INF = float("inf")
MARGIN = 16 * 2.0 ** -24


def plain(x, K, mode, bias, groups, top_groups, scale):
    """ids, weights and whether each token's choice is clear, in 64 bits on the CPU."""
    N, E = x.shape
    x = x.double()
    fit = (x > -INF) & ~x.isnan()
    x = torch.where(fit, x.clamp(max=torch.finfo(torch.float32).max), -INF)
    if mode & 0xFF == ex.EB_SIGMOID:
        s = torch.sigmoid(x)
    else:
        e = torch.where(fit, (x - x.max(1, keepdim=True).values).exp(), 0.0)
        s = e / e.sum(1, keepdim=True)
    judged = s + (0 if bias is None else bias.double())
    judged = torch.where(fit & ~judged.isnan(), judged, -INF)
    choice = x if bias is None else judged
    clear = torch.ones(N, dtype=torch.bool)

    def margin(sorted_values, k):
        """Whether every step down to the one after place k is wide."""
        v = sorted_values[:, :k + 1]
        return ((v[:, :-1] - v[:, 1:] > MARGIN) | (v[:, 1:] == -INF)).all(1)

    if groups > 1:
        pair = bool(mode & ex.EB_GROUP_PAIR)
        parts = (judged if pair else choice).view(N, groups, -1)
        worth = parts.topk(2, 2).values.sum(2) if pair else parts.max(2).values
        v, order = worth.sort(dim=1, descending=True, stable=True)
        if pair or bias is not None:
            at = torch.stack([v[:, top_groups - 1], v[:, min(top_groups, groups - 1)]], 1)
            clear &= margin(at, 1) if top_groups < groups else True
        keep = torch.zeros(N, groups, dtype=torch.bool).scatter_(1, order[:, :top_groups], True)
        choice = torch.where(keep.repeat_interleave(E // groups, 1), choice, -INF)
    v, ids = choice.sort(dim=1, descending=True, stable=True)
    if bias is not None:
        clear &= margin(v, K)
    ids = torch.where(v[:, :K] > -INF, ids[:, :K], -1)
    w = torch.where(ids >= 0, s.gather(1, ids.clamp(min=0)), 0.0)
    if mode & ex.EB_RENORMALIZE:
        # By logarithms: also where every score is below what 64 bits hold.
        log = torch.nn.functional.logsigmoid(x) if mode & 0xFF == ex.EB_SIGMOID else x
        log = torch.where(ids >= 0, log.gather(1, ids.clamp(min=0)), -INF)
        w = torch.where(ids >= 0, log.softmax(1), 0.0)
    return ids.int(), w * scale, clear


def grouping(ids, lo, hi):
    """offsets, tokens and slots of the pairs whose expert is in [lo, hi)."""
    N, K = ids.shape
    flat = ids.flatten().long()
    mine = (flat >= lo) & (flat < hi)
    pairs = mine.nonzero().flatten()
    order = pairs[flat[pairs].sort(stable=True).indices]
    offsets = torch.zeros(hi - lo + 1, dtype=torch.int32)
    offsets[1:] = torch.bincount(flat[pairs] - lo, minlength=hi - lo)[:hi - lo].cumsum(0) if hi > lo else 0
    tokens = torch.full((N * K,), -1, dtype=torch.int32)
    tokens[:order.numel()] = (order // K).int()
    slots = torch.full((N * K,), -1, dtype=torch.int32)
    slots[order] = torch.arange(order.numel(), dtype=torch.int32)
    return offsets, tokens, slots.view(N, K)


def check(x, K, device, mode=ex.EB_SOFTMAX, bias=None, groups=1, top_groups=1, scale=1.0, lo=0, hi=None, least_clear=0.9):
    N, E = x.shape
    hi = E if hi is None else hi
    r = ex.route(x if x.is_cuda else x.to(device), K, mode=mode, bias=None if bias is None else bias.to(device), groups=groups,
                 top_groups=top_groups, scale=scale, shard_lo=lo, shard_hi=hi)
    ids, w, clear = plain(x.cpu(), K, mode, bias, groups, top_groups, scale)
    got = r.ids.cpu()
    assert clear.float().mean() >= least_clear if N >= 8 else True
    assert torch.equal(got[clear], ids[clear])
    off = (r.weights.cpu().double() - w).abs()[clear]
    assert (off <= (E + 16) * 2.0 ** -24 * w[clear].abs() + 2.0 ** -126).all()
    assert (r.weights.cpu()[got < 0] == 0).all()
    for mine, want in zip((r.offsets, r.tokens, r.slots), grouping(got, lo, hi)):
        assert torch.equal(mine.cpu(), want)
    only = ex.route(x if x.is_cuda else x.to(device), K, mode=mode, bias=None if bias is None else bias.to(device), groups=groups,
                    top_groups=top_groups, scale=scale, grouped=False)
    assert torch.equal(only.ids, r.ids) and torch.equal(only.weights, r.weights) and only.slots is None
    return r


SIZES = [(N, E, K) for N in (1, 2, 3, 16, 31, 32, 33, 129, 1000, 5003)
         for E, K in ((1, 1), (2, 2), (8, 1), (17, 5), (32, 4), (64, 6), (100, 16), (160, 6), (256, 8), (257, 3), (513, 20), (1024, 64))
         if N * E <= 600_000]


@pytest.mark.parametrize("N,E,K", SIZES)
def test_softmax(N, E, K, device):
    g = torch.Generator().manual_seed(N * 7 + E)
    x = torch.randn(N, E, generator=g)
    check(x, K, device, ex.EB_SOFTMAX | (ex.EB_RENORMALIZE if N % 2 else 0), scale=1.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("function", [ex.EB_SOFTMAX, ex.EB_SIGMOID])
@pytest.mark.parametrize("E,K,groups,top_groups", [(16, 4, 1, 1), (40, 3, 5, 2), (64, 6, 8, 3), (96, 5, 3, 1), (256, 8, 8, 4), (256, 8, 32, 5),
                                                    (510, 20, 17, 6), (1024, 12, 32, 4)])
@pytest.mark.parametrize("judge", ["best", "pair", "bias", "bias+pair"])
def test_groups(dtype, function, E, K, groups, top_groups, judge, device):
    g = torch.Generator().manual_seed(E + K)
    x = torch.randn(203, E, generator=g).to(dtype)
    bias = 0.1 * torch.randn(E, generator=g) if "bias" in judge else None
    mode = function | ex.EB_RENORMALIZE | (ex.EB_GROUP_PAIR if "pair" in judge else 0)
    # Softmax scores of many experts crowd: more of their choices are close.
    check(x, K, device, mode, bias, groups, top_groups, 2.5, lo=E // 4, hi=E // 2, least_clear=0.5)


def test_ties_go_to_the_lowest_id(device):
    x = torch.zeros(70, 96)
    check(x, 9, device)
    x[:, 50:60] = 1.0
    x[::3, 95] = 1.0
    x[::5, 3] = -0.0
    check(x, 14, device, ex.EB_SIGMOID | ex.EB_RENORMALIZE)
    check(x, 14, device, ex.EB_SOFTMAX, groups=8, top_groups=3)


@pytest.mark.parametrize("function", [ex.EB_SOFTMAX, ex.EB_SIGMOID])
def test_scores_that_cannot_be_chosen(function, device):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(67, 48, generator=g)
    x[0] = -INF
    x[1] = float("nan")
    x[2, 3:] = -INF
    x[3, :40] = float("nan")
    x[4, 7] = INF
    x[5, [9, 30]] = INF
    x[6] = INF
    x[7] = torch.finfo(torch.float32).min
    x[8] = torch.finfo(torch.float32).max
    x[9] = -200.0  # sigmoid: every score is zero
    x[10, :] = -INF
    x[10, 47] = 0.0
    for mode in (function, function | ex.EB_RENORMALIZE):
        r = check(x, 5, device, mode)
        assert torch.isfinite(r.weights).all()
        check(x, 5, device, mode, groups=6, top_groups=2)
    r = check(x, 5, device, function, lo=8, hi=8)
    assert r.offsets.tolist() == [0] and (r.slots == -1).all()


def test_bias_with_nan_and_infinity(device):
    x = torch.zeros(5, 20)
    bias = torch.linspace(-1, 1, 20)
    bias[19], bias[18], bias[17] = float("nan"), INF, -INF
    r = ex.route(x.to(device), 20, mode=ex.EB_SIGMOID, bias=bias.to(device))
    assert r.ids[0].tolist() == [18] + list(range(16, -1, -1)) + [-1, -1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_scores(dtype, device):
    big = torch.randn(300, 150, device=device).to(dtype)
    check(big[5:250, 7:77], 6, device)
    check(big[::2, 1:130], 6, device)
    check(torch.randn(1, 64, device=device).to(dtype).expand(9, 64).contiguous()[:1], 3, device)


def test_no_tokens(device):
    r = ex.route(torch.empty(0, 32, device=device), 4, shard_lo=8, shard_hi=24)
    assert r.ids.shape == (0, 4) and r.offsets.tolist() == [0] * 17


def test_all_tokens_to_one_expert(device):
    x = torch.zeros(4097, 64)
    x[:, 63] = 5.0
    r = check(x, 1, device)
    assert r.offsets[-2].item() == 0 and r.offsets[-1].item() == 4097


def test_captured_into_a_graph(device):
    """Replays give what eager calls give, with other work between them."""
    for N in (3, 700):
        x = torch.randn(N, 96, device=device)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            ex.route(x, 6)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = ex.route(x, 6)
        for seed in range(4):
            x.copy_(torch.randn(N, 96, generator=torch.Generator().manual_seed(seed)))
            graph.replay()
            torch.cuda.synchronize()
            want = ex.route(x, 6)
            for a, b in zip(r, want):
                assert torch.equal(a, b)


def test_on_another_stream(device):
    side = torch.cuda.Stream()
    x = torch.randn(2000, 64, device=device)
    want = ex.route(x, 4)
    side.wait_stream(torch.cuda.current_stream())
    got = [ex.route(x, 4, stream=side) for _ in range(3)]
    side.synchronize()
    for r in got:
        for a, b in zip(r, want):
            assert torch.equal(a, b)


def test_refusals(device):
    x = torch.zeros(4, 32, device=device)
    for kw, code in ((dict(top=33), eb.EB_ERR_INVALID), (dict(top=0), eb.EB_ERR_INVALID), (dict(top=2, groups=5), eb.EB_ERR_INVALID),
                     (dict(top=2, groups=4, top_groups=5), eb.EB_ERR_INVALID), (dict(top=2, mode=7), eb.EB_ERR_INVALID),
                     (dict(top=2, mode=ex.EB_GROUP_PAIR, groups=32), eb.EB_ERR_INVALID),
                     (dict(top=2, shard_lo=5, shard_hi=33), eb.EB_ERR_INVALID)):
        with pytest.raises(eb.EbError) as e:
            ex.route(x, **kw)
        assert e.value.code == code, kw
    with pytest.raises(ValueError):
        ex.route(x.double(), 2)
    with pytest.raises(ValueError):
        ex.route(x.cpu(), 2)
    with pytest.raises(ValueError):
        ex.route(x.t(), 2)
    with pytest.raises(ValueError):
        ex.route(x, 2, bias=torch.zeros(31, device=device))


def test_softmax_of_chosen_far_below_the_largest(device):
    """The bias keeps the largest score out; the others' shares of each other stay."""
    g = torch.Generator().manual_seed(8)
    for N in (5, 700):
        x = torch.randn(N, 40, generator=g)
        x[:, 11] = 200.0
        bias = torch.linspace(0, 1, 40)
        bias[11] = -9.0
        r = check(x, 6, device, ex.EB_SOFTMAX | ex.EB_RENORMALIZE, bias)
        assert (r.ids != 11).all() and (r.weights > 0).all()
        pair = torch.randn(N, 40, generator=g)
        pair[:, 13], pair[:, 12:16:2], pair[:, 15] = 150.0, -INF, -INF  # its group has no second
        r = check(pair, 5, device, ex.EB_SOFTMAX | ex.EB_RENORMALIZE | ex.EB_GROUP_PAIR, groups=10, top_groups=4, least_clear=0.0)
        assert (r.ids != 13).all() and (r.weights > 0).all()


@pytest.mark.parametrize("N,E,K,lo,hi", [(341, 64, 3, 0, 64), (342, 64, 3, 5, 40), (2048, 160, 6, 80, 100), (4096, 8, 4, 0, 8), (4095, 6, 4, 2, 3),
                                         (2047, 1024, 8, 0, 1024), (16384, 3, 1, 0, 3), (16385, 3, 1, 0, 3), (300, 80, 50, 7, 80)])
@pytest.mark.parametrize("skewed", [False, True])
def test_pairs_placed_by_several_workgroups(N, E, K, lo, hi, skewed, device):
    x = torch.randn(N, E, generator=torch.Generator().manual_seed(N))
    if skewed:  # runs of tokens with the same choice, and tokens without any
        x[:N // 2] = torch.arange(E, 0, -1.0)
        x[N // 2:N // 2 + 100] = -INF
    check(x, K, device, ex.EB_SOFTMAX | ex.EB_RENORMALIZE, lo=lo, hi=hi)
