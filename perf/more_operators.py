"""Timed calls of what trains a layer of experts: layer norm, 8-bit checkpoints, sorting by expert, weight gradients.

A training step of a mixture of experts over pooled lookups takes, beside the routing, quantisation
and products of inference:

  norm        a layer norm of the pooled vectors, its output in floating point or in 8 bits (e4m3 with
              a scale per 1 x 128), and the normalised values kept in 8 bits (``train.layer_norm``);
  norm_back   its gradients, from the input or from what was kept (``train.layer_norm_backward``);
  act         the experts' activation of values kept in 8 bits (``train.activation``);
  act_back    its gradient, from the same (``train.activation_backward``);
  dispatch    the tokens' rows sorted by expert (``train.dispatch``);
  combine     the experts' rows joined per token, with weights, and without them the gradient of the
              sorting (``train.combine``);
  combine_back  the gradients of the joining (``train.combine_backward``);
  gradient    an expert's weight gradient from output gradients and inputs, either in 8 bits
              (``train.weight_gradient``).

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
EPS = 1e-5

NORM = dict(op="norm", rows=2048, cols=1024, dtype="f32", affine=True, out="bf16", keep="none")
NORM_BACK = dict(op="norm_back", rows=2048, cols=1024, dtype="bf16", x="fp8", affine=True)
ACT = dict(op="act", rows=256, hidden=1024, act="silu_gate", x="fp8", out="fp8")
ACT_BACK = dict(op="act_back", rows=8192, hidden=1024, act="silu_gate", x="fp8", dtype="bf16", out="fp8")
SORT = dict(op="dispatch", tokens=2048, experts=32, top=4, shards=1, width=1024, dtype="bf16", out="bf16", weights=True)
GRADIENT = dict(op="gradient", tokens=2048, experts=1, top=1, gather=False, outer=1024, inner=1024, dy="bf16", x="fp8", out="f32")


def listed():
    c = lambda base, name, **kw: dict(base, name=name, **kw)  # noqa: E731
    return [
        # One request's pooled vector on its way to the experts: the smallest call, latency only.
        c(NORM, "norm_one", rows=1, out="fp8"),
        # The large batch over 26 tables of 128 columns in training: what backward needs is kept in 8 bits.
        c(NORM, "norm_batch", rows=16384, cols=3328, keep="fp8"),
        # A step of 8 tables of 189 columns, which no tile divides; half precision, the input itself kept.
        c(NORM_BACK, "norm_back_odd", cols=1512, dtype="f16", x="f16"),
        # The large batch's gradients, from 8 bits.
        c(NORM_BACK, "norm_back_batch", rows=16384, cols=3328),
        # 64 tokens' slots between an expert's two products.
        c(ACT, "act_few"),
        # The large batch's slots (4 of 64 experts) on the way back.
        c(ACT_BACK, "act_back_batch", rows=65536),
        # One GPU's share (of two) of a step's rows, of no round width, made ready to be sent.
        c(SORT, "dispatch_odd", shards=2, width=1512, dtype="f16"),
        # The large batch's experts joined,
        c(SORT, "combine_batch", op="combine", tokens=16384, experts=64),
        # and the gradients of that, in 8 bits for the products that follow.
        c(SORT, "combine_back_batch", op="combine_back", tokens=16384, experts=64, out="fp8"),
        # A dense layer of widths that no tile divides; nothing in 8 bits.
        c(GRADIENT, "gradient_odd", outer=1000, inner=1512, x="bf16"),
        # A step's second expert layer: few slots to an expert, 16-bit gradients,
        c(GRADIENT, "gradient_down", experts=32, top=4, outer=512, out="bf16"),
        # and the large batch's first one, from tokens where they stand: the largest call.
        c(GRADIENT, "gradient_up", tokens=16384, experts=64, top=4, gather=True, outer=2048, dy="fp8"),
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
    kind = rng.choice(["norm", "norm_back", "act", "act_back", "dispatch", "combine", "combine_back", "gradient", "gradient", "gradient"])
    wide = rng.choice(["f32", "f16", "bf16"])
    if kind in ("norm", "norm_back"):
        cols = _width(rng, 64, 4096)
        rows = _log_int(rng, 1, min(32768, 54_000_000 // cols))
        if kind == "norm":
            return dict(NORM, rows=rows, cols=cols, dtype=wide, affine=rng.random() < 0.7, out=rng.choice(["f32", "f16", "bf16", "fp8"]),
                        keep=rng.choice(["none", "statistics", "fp8"]))
        return dict(NORM_BACK, rows=rows, cols=cols, dtype=wide, x=rng.choice([wide, "fp8"]), affine=rng.random() < 0.7)
    if kind in ("act", "act_back"):
        hidden = _width(rng, 64, 4096)
        return dict(ACT if kind == "act" else ACT_BACK, rows=_log_int(rng, 1, min(65536, 65_000_000 // hidden)), hidden=hidden,
                    act=rng.choice(["silu_gate", "silu_gate", "relu"]), x=rng.choice(["fp8", "fp8", "bf16", "f32"]),
                    out=rng.choice(["fp8", "fp8", "f32", "f16", "bf16"]), **({"dtype": wide} if kind == "act_back" else {}))
    if kind != "gradient":
        width, top = _width(rng, 64, 4096), rng.randint(1, 8)
        case = dict(SORT, op=kind, tokens=_log_int(rng, 1, max(1, min(16384, 64_000_000 // (width * top)))), top=top, width=width, dtype=wide,
                    experts=_log_int(rng, 8, 64), shards=rng.choice([1, 1, 2, 4]), weights=kind == "combine_back" or rng.random() < 0.7)
        if kind == "dispatch":
            dtype = rng.choice([wide, "fp8"])
            return dict(case, weights=False, dtype=dtype, shards=1 if dtype == "fp8" else case["shards"])
        if kind == "combine_back":
            case["shards"] = 1
        return dict(case, out=rng.choice(["f32", "f16", "bf16"] + (["fp8"] if kind == "combine_back" else [])))
    dy, x = rng.choice([("bf16", "fp8"), ("fp8", "fp8"), ("fp8", "fp8"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "fp8")])
    case = dict(GRADIENT, dy=dy, x=x, out=rng.choice(["f32", "f32", "bf16", "f16"]), tokens=_log_int(rng, 1, 16384), inner=_width(rng, 64, 4096),
                outer=_width(rng, 64, 4096))
    if rng.random() < 0.6:
        case.update(experts=_log_int(rng, 4, 64), top=rng.randint(1, 4), gather=rng.random() < 0.5, inner=_width(rng, 64, 2048),
                    outer=_width(rng, 64, 2048))
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


def _quantized(x):
    """e4m3 values [rows, cols], rows a multiple of 16 bytes apart, and their scales [rows, blocks], a block's of all rows side by side."""
    rows, cols = x.shape
    pad = torch.zeros(rows, _blocks(cols) * BLOCK, device="cuda")
    pad[:, :cols] = x
    b = pad.view(rows, -1, BLOCK)
    s = (b.abs().amax(2) / MOST_FP8).clamp(min=LEAST_SCALE)
    q = (b / s[:, :, None]).view(rows, -1).to(torch.float8_e4m3fn)
    return q[:, :cols], s.t().contiguous().t()


def _held(x, dtype):
    """Values in a type, with their scales where that is 8 bits."""
    return _quantized(x) if dtype == "fp8" else (x.to(DTYPES[dtype]), None)


def _rows(g, rows, cols, size=1.0):
    """Rows whose sizes differ, as those of pooled vectors (by their bags' lengths) and of gradients (by their samples) do."""
    return torch.randn(rows, cols, generator=g, device="cuda") * (size * torch.rand(rows, 1, generator=g, device="cuda").add_(0.1))


def _routed(case, g):
    """A route of the case's tokens: slots by expert as ``experts.route`` gives them, those of this GPU's experts kept."""
    N, E, top = case["tokens"], case["experts"], case["top"]
    liked = torch.randn(N, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    chosen = torch.topk(liked, top, 1).indices.flatten()
    held = -(-E // case.get("shards", 1))
    of, pair = torch.sort(chosen, stable=True)
    used = int((of < held).sum())
    at = torch.arange(N * top, device="cuda")
    slots = torch.empty_like(at).scatter_(0, pair, torch.where(of < held, at, -1))
    offsets = torch.searchsorted(of, torch.arange(held + 1, device="cuda"))
    weights = torch.softmax(torch.randn(N, top, generator=g, device="cuda"), 1)
    return {"tokens": torch.where(of < held, pair // top, -1).int(), "slots": slots.view(N, top).int(), "weights": weights,
            "offsets": offsets.int(), "used": used, "slot_expert": of}


def prepare(case, seed):
    g, op = _generator(seed, 1), case["op"]
    state = {"case": case}
    if op in ("norm", "norm_back"):
        rows, cols = case["rows"], case["cols"]
        x = _rows(g, rows, cols) + 0.3 * torch.randn(rows, 1, generator=g, device="cuda")
        state["weight"] = 1 + 0.1 * torch.randn(cols, generator=g, device="cuda") if case["affine"] else None
        bias = 0.1 * torch.randn(cols, generator=g, device="cuda")
        if op == "norm":
            return dict(state, x=x.to(DTYPES[case["dtype"]]), bias=bias if case["affine"] else None)
        # What forward left: the input and its statistics, or the normalised values in 8 bits.
        x = x if case["x"] == "fp8" else x.to(DTYPES[case["x"]])
        wide = x.float()
        mean = wide.mean(1)
        rstd = 1 / torch.sqrt((wide - mean[:, None]).square().mean(1) + EPS)
        held = _quantized((wide - mean[:, None]) * rstd[:, None]) if case["x"] == "fp8" else (x, None)
        return dict(state, x=held[0], x_scales=held[1], mean=None if case["x"] == "fp8" else mean, rstd=rstd,
                    dy=_rows(g, rows, cols, 1e-2).to(DTYPES[case["dtype"]]))
    if op in ("act", "act_back"):
        gated = case["act"] == "silu_gate"
        v, s = _held(2 * _rows(g, case["rows"], case["hidden"] * (2 if gated else 1)), case["x"])
        dh = _rows(g, case["rows"], case["hidden"], 1e-2).to(DTYPES[case["dtype"]]) if op == "act_back" else None
        return dict(state, v=v, v_scales=s, dh=dh)
    state.update(_routed(case, g))
    N = case["tokens"]
    if op == "dispatch":
        x, s = _held(_rows(g, N, case["width"]), case["dtype"])
        # The buffer that is sent; its rows behind the last slot stay as they are.
        return dict(state, x=x, x_scales=s, room=None if s is not None else torch.zeros(N * case["top"], case["width"], dtype=x.dtype, device="cuda"))
    if op in ("combine", "combine_back"):
        state["y"] = _rows(g, N * case["top"], case["width"]).to(DTYPES[case["dtype"]])
        if not case["weights"]:
            state["weights"] = None
        if op == "combine_back":
            state["dout"] = _rows(g, N, case["width"], 1e-2).to(DTYPES[case["dtype"]])
        return state
    if case["experts"] == 1:
        state.update(offsets=None, tokens=None)
    else:  # the plain form's plan: every slot's place among its expert's
        counts = torch.diff(state["offsets"])
        state.update(place=torch.arange(N * case["top"], device="cuda") - state["offsets"][state["slot_expert"]], most=int(counts.max()))
    state["dy"], state["dy_scales"] = _held(_rows(g, N * case["top"], case["outer"], 1e-2), case["dy"])
    state["x"], state["x_scales"] = _held(_rows(g, N if case["gather"] else N * case["top"], case["inner"]), case["x"])
    if not case["gather"]:
        state["tokens"] = None
    return state


# ------------------------------------------------------------------------------- the calls


def _act_code(case):
    from paper_2512_05831_amd import experts as ex

    return ex.EB_ACT_SILU_GATE if case["act"] == "silu_gate" else ex.EB_ACT_RELU


def _own(s):
    from paper_2512_05831_amd import train

    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        r = train.layer_norm(s["x"], s["weight"], s["bias"], EPS, out_dtype=DTYPES[c["out"]], statistics=c["keep"] == "statistics",
                             checkpoint=c["keep"] == "fp8")
        return {k: v for k, v in r._asdict().items() if v is not None}
    if op == "norm_back":
        return train.layer_norm_backward(s["dy"], s["x"], s["rstd"], mean=s["mean"], x_scales=s["x_scales"], weight=s["weight"],
                                         parameters=c["affine"])
    if op == "act":
        return train.activation(s["v"], s["v_scales"], act=_act_code(c), out_dtype=DTYPES[c["out"]])
    if op == "act_back":
        return train.activation_backward(s["dh"], s["v"], s["v_scales"], act=_act_code(c), out_dtype=DTYPES[c["out"]])
    if op == "dispatch":
        return train.dispatch(s["x"], s["tokens"], s["x_scales"], out=s["room"])
    if op == "combine":
        return train.combine(s["y"], s["slots"], s["weights"], out_dtype=DTYPES[c["out"]])
    if op == "combine_back":
        r = train.combine_backward(s["dout"], s["y"], s["slots"], s["weights"], out_dtype=DTYPES[c["out"]])
        return {k: v for k, v in r._asdict().items() if v is not None}
    return train.weight_gradient(s["dy"], s["x"], offsets=s["offsets"], tokens=s["tokens"], dy_scales=s["dy_scales"], x_scales=s["x_scales"],
                                 out_dtype=DTYPES[c["out"]])


def _wide(x, scales):
    """The values that a type holds, in 32 bits."""
    x = x.float()
    return x if scales is None else x * scales.repeat_interleave(BLOCK, 1)[:, :x.shape[1]]


def _narrow(x, dtype):
    """Rounded to a type once; for 8 bits with the scales."""
    if dtype != "fp8":
        return (x.to(DTYPES[dtype]),)
    rows, cols = x.shape
    pad = torch.zeros(rows, _blocks(cols) * BLOCK, device=x.device)
    pad[:, :cols] = x
    b = pad.view(rows, -1, BLOCK)
    s = (b.abs().amax(2) / MOST_FP8).clamp(min=LEAST_SCALE)
    return (b / s[:, :, None]).view(rows, -1)[:, :cols].to(torch.float8_e4m3fn), s


def _one_or_two(t):
    return t if len(t) > 1 else t[0]


def _plain_norm(s):
    c, x = s["case"], s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = 1 / torch.sqrt(x.square().mean(1) + EPS)
    x = x * rstd[:, None]
    out = dict(zip(("y", "y_scales"), _narrow(x * s["weight"] + s["bias"] if c["affine"] else x, c["out"])))
    if c["keep"] == "statistics":
        out.update(mean=mean, rstd=rstd)
    elif c["keep"] == "fp8":
        out.update(zip(("kept", "kept_scales"), _narrow(x, "fp8")), rstd=rstd)
    return out


def _plain_norm_back(s):
    c, dy, x, r = s["case"], s["dy"].float(), _wide(s["x"], s["x_scales"]), s["rstd"][:, None]
    if s["mean"] is not None:
        x = (x - s["mean"][:, None]) * r
    g = dy if s["weight"] is None else dy * s["weight"]
    dx = r * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True))
    return dx.to(DTYPES[c["dtype"]]), *(((dy * x).sum(0), dy.sum(0)) if c["affine"] else (None, None))


def _plain_act(s):
    c, v = s["case"], _wide(s["v"], s["v_scales"])
    if c["act"] == "relu":
        return _one_or_two(_narrow(v.clamp(min=0), c["out"]))
    g, u = v[:, :c["hidden"]], v[:, c["hidden"]:]
    return _one_or_two(_narrow(g / (1 + torch.exp(-g)) * u, c["out"]))


def _plain_act_back(s):
    c, v, dh = s["case"], _wide(s["v"], s["v_scales"]), s["dh"].float()
    if c["act"] == "relu":
        return _one_or_two(_narrow(torch.where(v > 0, dh, 0.0), c["out"]))
    g, u = v[:, :c["hidden"]], v[:, c["hidden"]:]
    p = 1 / (1 + torch.exp(-g))
    return _one_or_two(_narrow(torch.cat([dh * u * p * (1 + g * (1 - p)), dh * g * p], 1), c["out"]))


def _plain_combine(s):
    rows = torch.where((s["slots"] >= 0)[:, :, None], s["y"].float()[s["slots"].clamp(min=0).long()], 0.0)
    return (rows if s["weights"] is None else rows * s["weights"][:, :, None]).sum(1).to(DTYPES[s["case"]["out"]])


def _plain_combine_back(s):
    c, dout, slots = s["case"], s["dout"].float(), s["slots"]
    rows = dout[s["tokens"].long()]
    weight = torch.empty(len(rows), device="cuda")
    weight[slots.flatten().long()] = s["weights"].flatten()
    dots = (rows * s["y"].float()).sum(1)
    return dict(zip(("dy", "dy_scales"), _narrow(rows * weight[:, None], c["out"])), dweights=dots[slots.long()])


def _plain_gradient(s):
    c, dy, x = s["case"], _wide(s["dy"], s["dy_scales"]), _wide(s["x"], s["x_scales"])
    if s["tokens"] is not None:
        x = x[s["tokens"].long()]
    if s["offsets"] is None:
        return (dy.t() @ x).to(DTYPES[c["out"]])
    # Every expert's slots side by side, filled up to the most that one has.
    left = torch.zeros(c["experts"], s["most"], c["outer"], device="cuda")
    right = torch.zeros(c["experts"], s["most"], c["inner"], device="cuda")
    left[s["slot_expert"], s["place"]] = dy
    right[s["slot_expert"], s["place"]] = x
    return torch.bmm(left.transpose(1, 2), right).to(DTYPES[c["out"]])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "norm":
        return _plain_norm(state)
    if op == "norm_back":
        return _plain_norm_back(state)
    if op == "act":
        return _plain_act(state)
    if op == "act_back":
        return _plain_act_back(state)
    if op == "dispatch":
        at = state["tokens"].long()
        if state["x_scales"] is not None:
            return state["x"][at], state["x_scales"][at]
        return torch.where((at >= 0)[:, None], state["x"][at.clamp(min=0)], state["room"])
    if op == "combine":
        return _plain_combine(state)
    if op == "combine_back":
        return _plain_combine_back(state)
    return _plain_gradient(state)


# ------------------------------------------------------------------------------- what they have to do


def _bytes(rows, cols, dtype):
    """A matrix, with its scales where it is in 8 bits."""
    return rows * cols * SIZES[dtype] + (4 * rows * _blocks(cols) if dtype == "fp8" else 0)


def work(case):
    op = case["op"]
    if op in ("norm", "norm_back"):
        rows, cols, affine = case["rows"], case["cols"], 8 * case["cols"] if case["affine"] else 0
        if op == "norm":
            kept = {"none": 0, "statistics": 8 * rows, "fp8": 4 * rows + _bytes(rows, cols, "fp8")}[case["keep"]]
            return {"bytes": _bytes(rows, cols, case["dtype"]) + _bytes(rows, cols, case["out"]) + kept + affine, "flops": 8.0 * rows * cols}
        return {"bytes": 2 * _bytes(rows, cols, case["dtype"]) + _bytes(rows, cols, case["x"]) + (4 if case["x"] == "fp8" else 8) * rows
                + 3 * affine // 2, "flops": 14.0 * rows * cols}
    if op in ("act", "act_back"):
        rows, hidden, both = case["rows"], case["hidden"], case["hidden"] * (2 if case["act"] == "silu_gate" else 1)
        if op == "act":
            return {"bytes": _bytes(rows, both, case["x"]) + _bytes(rows, hidden, case["out"]), "flops": 6.0 * rows * hidden}
        return {"bytes": _bytes(rows, both, case["x"]) + _bytes(rows, hidden, case["dtype"]) + _bytes(rows, both, case["out"]),
                "flops": 12.0 * rows * hidden}
    N, pairs, W = case["tokens"], case["tokens"] * case["top"], case.get("width")
    if op == "gradient":
        E, out, K = case["experts"], case["outer"], case["inner"]
        return {"bytes": _bytes(pairs, out, case["dy"]) + _bytes(N if case["gather"] else pairs, K, case["x"]) + E * out * K * SIZES[case["out"]]
                + (4 * (E + 1) if E > 1 else 0) + (4 * pairs if case["gather"] else 0), "flops": 2.0 * pairs * out * K}
    # Of several GPUs' experts one has its share of the pairs.
    used = pairs * -(-case["experts"] // case["shards"]) // case["experts"]
    weights = 4 * pairs if case["weights"] else 0
    if op == "dispatch":
        return {"bytes": _bytes(min(N, used), W, case["dtype"]) + _bytes(used, W, case["dtype"]) + 4 * used, "flops": 0.0}
    if op == "combine":
        return {"bytes": _bytes(used, W, case["dtype"]) + _bytes(N, W, case["out"]) + 4 * pairs + weights, "flops": 2.0 * used * W}
    return {"bytes": _bytes(N, W, case["dtype"]) + _bytes(used, W, case["dtype"]) + _bytes(used, W, case["out"]) + 8 * pairs + weights,
            "flops": 3.0 * used * W}


# ------------------------------------------------------------------------------- the definitions, in 64 bits


def _values(x, scales):
    x = x.double()
    if scales is not None:
        x = x * scales.double()[:, torch.arange(x.shape[1], device=x.device) // BLOCK]
    return x


def _eight(v):
    """e4m3 numbers (nearest, ties to even) and scales of 64-bit rows."""
    rows, cols = v.shape
    most = torch.nn.functional.pad(v.abs(), (0, -cols % BLOCK)).view(rows, -1, BLOCK).amax(2)
    s = (most / MOST_FP8).clamp(min=LEAST_SCALE)
    q = v / s[:, torch.arange(cols, device=v.device) // BLOCK]
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(q / step) * step, s


def _exact_norm(s):
    c = s["case"]
    x = s["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    r = (var + EPS).rsqrt()
    n = (x - mean[:, None]) * r[:, None]
    y = n if s["weight"] is None else torch.addcmul(s["bias"].double(), n, s["weight"].double())
    out = dict(zip(("y", "y_scales"), _eight(y) if c["out"] == "fp8" else (y,)))
    if c["keep"] != "none":
        out["rstd"] = r
    if c["keep"] == "statistics":
        out["mean"] = mean
    if c["keep"] == "fp8":
        out["kept"], out["kept_scales"] = _eight(n)
    return out


def _exact_norm_back(s):
    dy, n, r = s["dy"].double(), _values(s["x"], s["x_scales"]), s["rstd"].double()
    if s["mean"] is not None:
        n = (n - s["mean"].double()[:, None]) * r[:, None]
    g = dy if s["weight"] is None else dy * s["weight"].double()
    cols = g.shape[1]
    dx = (g - (g.sum(1) / cols)[:, None] - n * (torch.linalg.vecdot(g, n) / cols)[:, None]) * r[:, None]
    if not s["case"]["affine"]:
        return dx, None, None
    return dx, torch.linalg.vecdot(dy, n, dim=0), dy.sum(0)


def _exact_act(s):
    c, v = s["case"], _values(s["v"], s["v_scales"])
    if c["act"] == "relu":
        h = torch.relu(v)
    else:
        g, u = v.chunk(2, 1)
        h = g * torch.sigmoid(g) * u
    return _eight(h) if c["out"] == "fp8" else h


def _exact_act_back(s):
    c, v, dh = s["case"], _values(s["v"], s["v_scales"]), s["dh"].double()
    if c["act"] == "relu":
        dv = dh * (v > 0)
    else:
        g, u = v.chunk(2, 1)
        p = torch.sigmoid(g)
        dv = torch.cat([dh * u * (p + g * p * torch.sigmoid(-g)), dh * g * p], 1)
    return _eight(dv) if c["out"] == "fp8" else dv


def _exact_sort(s):
    c = s["case"]
    if c["op"] == "dispatch":
        at = s["tokens"].long()
        if s["x_scales"] is not None:
            return s["x"].double()[at], s["x_scales"].double()[at]
        rows = s["room"].double()
        rows[:s["used"]] = s["x"].double()[at[:s["used"]]]
        return rows
    y, slots = s["y"].double(), s["slots"].long()
    mine = slots >= 0
    token, k = mine.nonzero(as_tuple=True)
    slot = slots[token, k]
    w = torch.ones(slots.shape, dtype=torch.float64, device="cuda") if s["weights"] is None else s["weights"].double()
    if c["op"] == "combine":
        out = torch.zeros(c["tokens"], c["width"], dtype=torch.float64, device="cuda")
        return out.index_add_(0, token, y[slot] * w[token, k, None])
    dout = s["dout"].double()
    dy = torch.empty_like(y)
    dy[slot] = dout[token] * w[token, k, None]
    dweights = torch.zeros_like(w)
    dweights[token, k] = torch.linalg.vecdot(dout[token], y[slot])
    return dict(zip(("dy", "dy_scales"), _eight(dy) if c["out"] == "fp8" else (dy,)), dweights=dweights)


def _exact_gradient(s):
    dy, x = _values(s["dy"], s["dy_scales"]), _values(s["x"], s["x_scales"])
    if s["offsets"] is None:
        return torch.mm(dy.t(), x)
    bounds = s["offsets"].tolist()
    dw = torch.zeros(len(bounds) - 1, dy.shape[1], x.shape[1], dtype=torch.float64, device="cuda")
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        rows = x[a:b] if s["tokens"] is None else x[s["tokens"][a:b].long()]
        torch.mm(dy[a:b].t(), rows, out=dw[e])
    return dw


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "gradient":
        return _exact_gradient(s)
    if op in ("dispatch", "combine", "combine_back"):
        return _exact_sort(s)
    return {"norm": _exact_norm, "norm_back": _exact_norm_back, "act": _exact_act, "act_back": _exact_act_back}[op](s)
