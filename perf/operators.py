"""Timed calls of the experts' operators: routing, 8-bit quantisation and the block-scaled product.

A mixture of experts over pooled lookups is three operators of this package, and the weighted
pooled lookup that joins the experts' rows again:

  route     one row of scores per token: the top experts, their weights, and the chosen (token,
            expert) pairs grouped by expert (``experts.route``);
  quantize  8-bit floating point (e4m3) with one fp32 scale per 1 x 128 values of a row, or per
            128 x 128 of a weight matrix (``experts.quantize_fp8``);
  product   rows times an expert's weights, both 8 bits with those scales, with a bias, a ReLU or a
            gated SiLU, and an output in floating point or in 8 bits again (``experts.product``).

``listed`` names fixed calls, ``draw`` gives further ones from the same ranges.  ``run`` makes them
through the package where ``own`` is true, else in elementary torch operations of 32 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
SIZES = {"f32": 4, "f16": 2, "bf16": 2, "fp8": 1}
BLOCK = 128
MOST_FP8 = 448.0
LEAST_SCALE = 2.0 ** -126

ROUTE = dict(op="route", tokens=256, experts=64, top=4, score="softmax", bias=False, groups=1, top_groups=1,
             pair=False, renormalize=True, scale=1.0, dtype="f32", padded=0.0, shards=1)
QUANTIZE = dict(op="quantize", matrices=1, rows=2048, cols=1024, dtype="f32", block_rows=1)
PRODUCT = dict(op="product", tokens=256, experts=1, top=1, gather=False, inner=1024, outer=1024, act="none",
               bias=False, out="bf16")


def listed():
    r = lambda name, **kw: dict(ROUTE, name=name, **kw)  # noqa: E731
    q = lambda name, **kw: dict(QUANTIZE, name=name, **kw)  # noqa: E731
    p = lambda name, **kw: dict(PRODUCT, name=name, **kw)  # noqa: E731
    return [
        # One request: the smallest call, latency only.
        r("route_one", tokens=1, experts=32),
        # A serving batch of half-precision scores, plain softmax weights.
        r("route_serving", tokens=256, top=6, renormalize=False, dtype="bf16"),
        # One GPU's mini-batch, an expert count that is no power of two, experts in groups, some padded rows, and
        # the experts of one GPU of eight kept.
        r("route_grouped_shard", tokens=2048, experts=160, top=6, groups=8, top_groups=3, dtype="f16", scale=16.0,
          renormalize=False, padded=0.05, shards=8),
        # The large inference batch with sigmoid scores, a bias for balance and pairs of experts judging a group.
        r("route_batch", tokens=16384, experts=256, top=8, score="sigmoid", bias=True, groups=8, top_groups=4,
          pair=True, scale=2.5),
        # Pooled vectors of one batch of 8 tables of 128 columns,
        q("quantize_step"),
        # and of the large batch of 26 tables.
        q("quantize_batch", rows=16384, cols=3328),
        # One request through a dense layer: latency and the weights' bytes.
        p("product_one", tokens=1, outer=2048),
        # Widths that no tile divides (8 tables of 189 columns), with a bias and a ReLU, fp32 output.
        p("product_odd", tokens=2048, inner=1512, outer=1000, act="relu", bias=True, out="f32"),
        # The large batch's first dense layer over 26 tables: the largest product.
        p("product_batch", tokens=16384, inner=3328, outer=4096),
        # A serving batch's first expert layer: every expert's weights are read for a few rows each.
        p("experts_serving", tokens=64, experts=32, top=4, gather=True, outer=2048, act="silu_gate", out="fp8"),
        # The large batch's first expert layer, gated, 8 bits out,
        p("experts_up", tokens=16384, experts=64, top=4, gather=True, outer=2048, act="silu_gate", out="fp8"),
        # and its second, on the slots in order.
        p("experts_down", tokens=16384, experts=64, top=4),
    ]


# ------------------------------------------------------------------------------- drawn cases


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width that tiles divide, or one that no tile does."""
    if rng.random() < 0.5:
        return rng.choice([n for n in (128, 256, 384, 512, 640, 768, 1024, 1280, 1664, 2048, 2560, 3328, 4096) if lo <= n <= hi])
    n = _log_int(rng, lo, hi)
    return n if n % BLOCK else n + 1


def draw(rng):
    kind = rng.choice(["route", "route", "quantize", "product", "product", "experts", "experts"])
    if kind == "route":
        tokens = _log_int(rng, 1, 16384)
        groups = rng.choice([1, 1, 4, 8])
        experts = rng.choice([16, 32, 64, 128, 256])
        if rng.random() < 0.5:
            experts = groups * rng.randint(max(2, 8 // groups), 256 // groups)
        sigmoid = rng.random() < 0.5
        top_groups = rng.randint(1, max(1, groups // 2))
        top = rng.randint(1, min(8, experts // groups * top_groups))
        return dict(ROUTE, tokens=tokens, experts=experts, top=top, groups=groups, top_groups=top_groups,
                    score="sigmoid" if sigmoid else "softmax", bias=sigmoid and rng.random() < 0.7,
                    pair=sigmoid and groups > 1 and rng.random() < 0.5, renormalize=rng.random() < 0.6,
                    scale=rng.choice([1.0, 2.5]), dtype=rng.choice(["f32", "f16", "bf16"]),
                    padded=rng.choice([0.0, 0.0, 0.1]), shards=rng.choice([1, 1, 2, 4]))
    if kind == "quantize":
        dtype = rng.choice(["f32", "f16", "bf16"])
        cols = _width(rng, 64, 4096)
        if rng.random() < 0.3:  # an expert layer's weights
            return dict(QUANTIZE, matrices=rng.randint(1, 32), rows=_width(rng, 128, 1024), cols=cols, dtype=dtype,
                        block_rows=BLOCK)
        return dict(QUANTIZE, rows=_log_int(rng, 1, min(32768, 54_000_000 // cols)), cols=cols, dtype=dtype)
    act = rng.choice(["none", "none", "relu", "silu_gate"])
    case = dict(PRODUCT, act=act, bias=rng.random() < 0.3, out=rng.choice(["f32", "f16", "bf16", "bf16", "fp8"]),
                inner=_width(rng, 64, 4096), outer=_width(rng, 64, 4096))
    if kind == "product":
        case.update(tokens=_log_int(rng, 1, 16384))
    else:
        case.update(experts=_log_int(rng, 4, 64), gather=rng.random() < 0.5, tokens=_log_int(rng, 1, 16384),
                    inner=_width(rng, 64, 2048), outer=_width(rng, 64, 2048))
        case.update(top=rng.randint(1, 4))
    if act == "silu_gate":
        case["outer"] += case["outer"] % 2  # two halves
    while 2.0 * case["tokens"] * case["top"] * case["inner"] * case["outer"] > 2.5e11:
        case["tokens"] = max(1, case["tokens"] * 2 // 3)
    return case


# ------------------------------------------------------------------------------- inputs


def _blocks(n):
    return -(-n // BLOCK)


def _generator(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 16 + what)
    return g


def _scores(case, seed):
    """Router scores: tokens differ, some experts are liked more, padded tokens are all -inf."""
    g = _generator(seed, 0)
    N, E = case["tokens"], case["experts"]
    x = torch.randn(N, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    if case.get("padded"):
        x[torch.rand(N, generator=g, device="cuda") < case["padded"]] = -math.inf
    return x.to(DTYPES[case.get("dtype", "f32")])


def _quantized_rows(x):
    """e4m3 values [rows, cols] and their scales [rows, blocks] (a block's scales of all rows side by side)."""
    rows, cols = x.shape
    pad = torch.zeros(rows, _blocks(cols) * BLOCK, device="cuda")
    pad[:, :cols] = x
    b = pad.view(rows, -1, BLOCK)
    s = (b.abs().amax(2) / MOST_FP8).clamp(min=LEAST_SCALE)
    q = (b / s[:, :, None]).view(rows, -1).to(torch.float8_e4m3fn)
    return q[:, :cols], s.t().contiguous().t()


def prepare(case, seed):
    g = _generator(seed, 1)
    if case["op"] == "route":
        bias = 0.05 * torch.randn(case["experts"], generator=g, device="cuda") if case["bias"] else None
        held = -(-case["experts"] // case["shards"])
        return {"case": case, "scores": _scores(case, seed), "bias": bias,
                "lo": 0 if case["shards"] == 1 else held * (case["shards"] // 2), "held": held}
    if case["op"] == "quantize":
        # Pooled sums: the rows' sizes follow their bags' lengths.
        x = torch.randn(case["matrices"], case["rows"], case["cols"], generator=g, device="cuda")
        x *= 0.01 * torch.rand(case["matrices"], case["rows"], 1, generator=g, device="cuda").mul_(10).add_(0.1)
        return {"case": case, "x": (x if case["block_rows"] > 1 else x[0]).to(DTYPES[case["dtype"]])}
    N, E, K, out = case["tokens"], case["experts"], case["inner"], case["outer"]
    S = N * case["top"]
    state = {"case": case, "offsets": None, "tokens": None, "slot_expert": None, "place": None, "most": S}
    if E > 1:  # the route of these tokens, grouped by expert
        chosen = torch.topk(_scores(dict(case, padded=0.0), seed), case["top"], 1).indices.flatten()
        of, pair = torch.sort(chosen, stable=True)
        counts = torch.bincount(of, minlength=E)
        offsets = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
        torch.cumsum(counts, 0, out=offsets[1:])
        # The plain form's plan: every slot's expert, and its place among that expert's.
        state.update(offsets=offsets.int(), tokens=(pair // case["top"]).int() if case["gather"] else None, slot_expert=of,
                     place=torch.arange(S, device="cuda") - offsets[of], most=int(counts.max()))
    x = torch.randn(N if E > 1 and case["gather"] else S, K, generator=g, device="cuda")
    state["x"], state["x_scales"] = _quantized_rows(x * torch.rand(x.shape[0], 1, generator=g, device="cuda").add_(0.1))
    # Weights of a trained layer's size, as 8-bit values under scales that differ from block to block.  Under a
    # gate each half of the rows is blocked on its own.
    halves = 2 if case["act"] == "silu_gate" else 1
    pitch = -(-K // 16) * 16
    w = torch.empty(E, out, pitch, dtype=torch.float8_e4m3fn, device="cuda")
    for e in range(E):
        w[e] = (torch.randn(out, pitch, generator=g, device="cuda") * 100).clamp_(-MOST_FP8, MOST_FP8).to(w.dtype)
    state["w"] = w[:, :, :K] if E > 1 else w[0, :, :K]
    s = torch.rand(E, halves * _blocks(out // halves), _blocks(K), generator=g, device="cuda").add_(0.5).mul_(0.01 / math.sqrt(K))
    state["w_scales"] = s if E > 1 else s[0]
    state["bias"] = torch.randn(E, out, generator=g, device="cuda").mul_(0.1) if case["bias"] else None
    if state["bias"] is not None and E == 1:
        state["bias"] = state["bias"][0]
    return state


# ------------------------------------------------------------------------------- the calls


def _own_route(s):
    from paper_2512_05831_amd import experts as ex

    c = s["case"]
    mode = ex.EB_SIGMOID if c["score"] == "sigmoid" else ex.EB_SOFTMAX
    mode |= (ex.EB_RENORMALIZE if c["renormalize"] else 0) | (ex.EB_GROUP_PAIR if c["pair"] else 0)
    hi = min(c["experts"], s["lo"] + s["held"])
    return ex.route(s["scores"], c["top"], mode=mode, bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"],
                    scale=c["scale"], shard_lo=s["lo"], shard_hi=hi)._asdict()


def _own_product(s):
    from paper_2512_05831_amd import experts as ex

    c = s["case"]
    act = {"none": ex.EB_ACT_NONE, "relu": ex.EB_ACT_RELU, "silu_gate": ex.EB_ACT_SILU_GATE}[c["act"]]
    return ex.product(s["x"], s["x_scales"], s["w"], s["w_scales"], offsets=s["offsets"], tokens=s["tokens"],
                      bias=s["bias"], act=act, out_dtype=DTYPES[c["out"]])


def _plain_route(s):
    c, b = s["case"], s["bias"]
    N, E, K, G = c["tokens"], c["experts"], c["top"], c["groups"]
    x = s["scores"].float().clamp(max=torch.finfo(torch.float32).max)
    may = x > -math.inf
    x = torch.where(may, x, -math.inf)
    if c["score"] == "sigmoid":
        p = 1 / (1 + torch.exp(-x))
    else:
        e = torch.where(may, torch.exp(x - x.amax(1, keepdim=True)), 0.0)
        p = e / e.sum(1, keepdim=True)
    judged = torch.where(may, p if b is None else p + b, -math.inf)
    choice = x if b is None else judged
    if G > 1:
        if c["pair"]:
            of_group = torch.sort(judged.view(N, G, -1), dim=2, descending=True).values[:, :, :2].sum(2)
        else:
            of_group = choice.view(N, G, -1).amax(2)
        best = torch.sort(of_group, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros(N, G, dtype=torch.bool, device=x.device).scatter_(1, best, True)
        choice = torch.where(keep.repeat_interleave(E // G, 1), choice, -math.inf)
    value, ids = torch.sort(choice, dim=1, descending=True, stable=True)
    value, ids = value[:, :K], ids[:, :K]
    found = value > -math.inf
    w = torch.where(found, p.gather(1, ids), 0.0)
    if c["renormalize"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    ids = torch.where(found, ids, -1)
    # Grouping by expert: pairs of other shards, and those without an expert, sort behind.
    held = min(E, s["lo"] + s["held"]) - s["lo"]
    flat = ids.flatten() - s["lo"]
    flat = torch.where((flat >= 0) & (flat < held) & (ids.flatten() >= 0), flat, held)
    of, pair = torch.sort(flat, stable=True)
    offsets = torch.searchsorted(of, torch.arange(held + 1, device=x.device))
    mine = of < held
    at = torch.arange(N * K, device=x.device)
    slots = torch.empty_like(at).scatter_(0, pair, torch.where(mine, at, -1)).view(N, K)
    return {"ids": ids.int(), "weights": w * c["scale"], "offsets": offsets.int(),
            "tokens": torch.where(mine, pair // K, -1).int(), "slots": slots.int()}


def _plain_quantize(x, block_rows):
    """x: [matrices, rows, cols] in 32 bits, padded with zeros to whole blocks here."""
    m, rows, cols = x.shape
    rb, cb = -(-rows // block_rows), _blocks(cols)
    pad = torch.zeros(m, rb * block_rows, cb * BLOCK, device=x.device)
    pad[:, :rows, :cols] = x
    b = pad.view(m, rb, block_rows, cb, BLOCK)
    most = b.abs().amax((2, 4))
    s = torch.where(torch.isfinite(most), (most / MOST_FP8).clamp(min=LEAST_SCALE), math.nan)
    q = (b / s[:, :, None, :, None]).view(m, rb * block_rows, -1)[:, :rows, :cols]
    return q.to(torch.float8_e4m3fn), s


def _plain_product(s):
    c = s["case"]
    N, E, K, out = c["tokens"], c["experts"], c["inner"], c["outer"]
    x, w, ws = s["x"].float(), s["w"].float().view(E, out, -1), s["w_scales"].view(E, -1, _blocks(K))
    x = x * s["x_scales"].repeat_interleave(BLOCK, 1)[:, :K]
    half = out // 2 if c["act"] == "silu_gate" else out
    per_row = ws.view(E, out // half, -1, ws.shape[2]).repeat_interleave(BLOCK, 2)[:, :, :half].reshape(E, out, -1)
    w = (w * per_row.repeat_interleave(BLOCK, 2)[:, :, :K]).transpose(1, 2)
    if E > 1:  # every expert's rows side by side, filled up to the longest
        rows = x if s["tokens"] is None else x[s["tokens"].long()]
        full = torch.zeros(E, s["most"], K, device=x.device)
        full[s["slot_expert"], s["place"]] = rows
        y = torch.bmm(full, w)
        y = (y if s["bias"] is None else y + s["bias"][:, None])[s["slot_expert"], s["place"]]
    else:
        y = x @ w[0]
        y = y if s["bias"] is None else y + s["bias"]
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "silu_gate":
        y = y[:, :half] / (1 + torch.exp(-y[:, :half])) * y[:, half:]
    if c["out"] == "fp8":
        q, scales = _plain_quantize(y[None], 1)
        return q[0], scales[0]
    return y.to(DTYPES[c["out"]])


def run(state):
    c = state["case"]
    if c["op"] == "route":
        return _own_route(state) if own else _plain_route(state)
    if c["op"] == "product":
        return _own_product(state) if own else _plain_product(state)
    if own:
        from paper_2512_05831_amd import experts as ex

        return ex.quantize_fp8(state["x"], block_rows=c["block_rows"])
    x = state["x"].float()
    q, s = _plain_quantize(x if x.dim() == 3 else x[None], c["block_rows"])
    return (q, s) if x.dim() == 3 else (q[0], s[0])


# ------------------------------------------------------------------------------- what they have to do


def work(case):
    if case["op"] == "route":
        N, E, pairs = case["tokens"], case["experts"], case["tokens"] * case["top"]
        held = -(-E // case["shards"])
        return {"bytes": N * E * SIZES[case["dtype"]] + (4 * E if case["bias"] else 0) + 16 * pairs + 4 * (held + 1),
                "flops": 4.0 * N * E}
    if case["op"] == "quantize":
        rows, cols = case["matrices"] * case["rows"], case["cols"]
        scales = case["matrices"] * -(-case["rows"] // case["block_rows"]) * _blocks(cols)
        return {"bytes": rows * cols * (SIZES[case["dtype"]] + 1) + 4 * scales, "flops": 2.0 * rows * cols}
    S, E, K, out = case["tokens"] * case["top"], case["experts"], case["inner"], case["outer"]
    halves = 2 if case["act"] == "silu_gate" else 1
    read_rows = case["tokens"] if E > 1 and case["gather"] else S
    used = min(E, S)
    written = S * (out // halves)
    return {"bytes": read_rows * (K + 4 * _blocks(K)) + used * (out * K + 4 * halves * _blocks(out // halves) * _blocks(K))
            + (4 * used * out if case["bias"] else 0) + (4 * (E + 1) if E > 1 else 0) + (4 * S if E > 1 and case["gather"] else 0)
            + written * SIZES[case["out"]] + (4 * S * _blocks(out // halves) if case["out"] == "fp8" else 0),
            "flops": 2.0 * S * out * K}


# ------------------------------------------------------------------------------- the definitions, in 64 bits


def _exact_route(s):
    """Weights only: the whole numbers have no rounding."""
    c = s["case"]
    x = s["scores"].double()
    N, E, G = c["tokens"], c["experts"], c["groups"]
    masked = torch.isneginf(x)
    score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, 1)
    order = score if s["bias"] is None else score + s["bias"].double()
    order = order.masked_fill(masked, -math.inf)
    if G > 1:
        parts = order.reshape(N, G, E // G)
        rank = parts.topk(2, 2).values.sum(2) if c["pair"] else parts.max(2).values
        gone = torch.ones(N, G, dtype=torch.bool, device=x.device)
        gone[torch.arange(N, device=x.device)[:, None], rank.argsort(dim=1, descending=True, stable=True)[:, :c["top_groups"]]] = False
        order = parts.masked_fill(gone[:, :, None], -math.inf).reshape(N, E)
    ids = order.argsort(dim=1, descending=True, stable=True)[:, :c["top"]]
    w = torch.take_along_dim(score, ids, 1).masked_fill(torch.take_along_dim(order, ids, 1).isneginf(), 0.0)
    if c["renormalize"]:
        w = torch.nan_to_num(w / w.sum(1, keepdim=True), nan=0.0)
    return {"ids": None, "weights": w * c["scale"], "offsets": None, "tokens": None, "slots": None}


def _round_e4m3(v):
    """|v| <= 448 to the nearest e4m3 number, ties to even, in 64 bits."""
    exponent = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    return torch.round(v / step) * step


def _exact_fp8(y, block_rows):
    m, rows, cols = y.shape
    q = torch.empty_like(y)
    s = torch.empty(m, -(-rows // block_rows), _blocks(cols), dtype=torch.float64, device=y.device)
    for j in range(s.shape[2]):
        part = y[:, :, j * BLOCK:(j + 1) * BLOCK]
        most = part.abs().amax(2)
        if block_rows > 1:
            most = torch.nn.functional.pad(most, (0, -rows % block_rows)).view(m, -1, block_rows).amax(2)
        s[:, :, j] = (most / MOST_FP8).clamp(min=LEAST_SCALE)
        q[:, :, j * BLOCK:(j + 1) * BLOCK] = _round_e4m3(part / s[:, :, j].repeat_interleave(block_rows, 1)[:, :rows, None])
    return q, s


def _exact_product(s):
    c = s["case"]
    S, E, K, out = c["tokens"] * c["top"], c["experts"], c["inner"], c["outer"]
    gated = c["act"] == "silu_gate"
    half = out // 2 if gated else out
    block = torch.arange(K, device="cuda") // BLOCK
    line = torch.cat([torch.arange(half, device="cuda") // BLOCK + i * _blocks(half) for i in range(out // half)])
    bounds = [0, S] if E == 1 else s["offsets"].tolist()
    y = torch.empty(S, half, dtype=torch.float64, device="cuda")
    for e in range(E):
        w, ws = (s["w"], s["w_scales"]) if E == 1 else (s["w"][e], s["w_scales"][e])
        w = w.double() * ws.double()[line][:, block]
        for a in range(bounds[e], bounds[e + 1], 4096):
            b = min(a + 4096, bounds[e + 1])
            rows = torch.arange(a, b, device="cuda") if s["tokens"] is None else s["tokens"][a:b].long()
            v = (s["x"][rows.min():rows.max() + 1].double()[rows - rows.min()] * s["x_scales"][rows].double()[:, block]) @ w.t()
            if s["bias"] is not None:
                v = v + (s["bias"] if E == 1 else s["bias"][e]).double()
            if c["act"] == "relu":
                v = torch.relu(v)
            if gated:
                v = v[:, :half] * torch.sigmoid(v[:, :half]) * v[:, half:]
            y[a:b] = v
    if c["out"] != "fp8":
        return y
    q, scales = _exact_fp8(y[None], 1)
    return q[0], scales[0]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        return _exact_route(s)
    if case["op"] == "product":
        return _exact_product(s)
    x = s["x"].double()
    q, scales = _exact_fp8(x if x.dim() == 3 else x[None], case["block_rows"])
    return (q, scales) if x.dim() == 3 else (q[0], scales[0])
