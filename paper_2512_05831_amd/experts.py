"""Python binding of the C ABI in ``include/eb_experts.h`` (ctypes, marshalling only).

A mixture of experts over pooled lookups: ``route`` chooses every token's experts
and groups the chosen pairs by expert, ``quantize_fp8`` brings vectors and weights
to 8 bits with a scale per block of 128, ``product`` multiplies each slot's vector
with its expert's weights.  ``eb_route_experts``, ``eb_quantize_fp8`` and
``eb_expert_product`` are the C calls under their own names, with device addresses
as ints.  There is no fallback: every step runs in ``libeb.so``.

``ExpertLayer`` runs them together: the experts' two layers for a batch of
vectors, joined per token by a weighted pooled lookup (``EmbeddingBagTables``).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from . import eb
from .eb import EB_BF16, EB_F16, EB_F32, EB_SUM, EbError, _check, _same_device, _stream_ptr

EB_FP8 = 3
EB_SOFTMAX, EB_SIGMOID = 0, 1
EB_RENORMALIZE, EB_GROUP_PAIR = 0x100, 0x200
EB_ACT_NONE, EB_ACT_RELU, EB_ACT_SILU_GATE = 0, 1, 2
BLOCK = 128

_lib = None


def library() -> ctypes.CDLL:
    """``eb.library()`` with the experts' functions declared."""
    global _lib
    if _lib is None:
        lib = eb.library()
        p, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        lib.eb_route_experts_workspace.argtypes = [i64, i32, i32, i32, ctypes.POINTER(size)]
        lib.eb_route_experts_workspace.restype = ctypes.c_int
        lib.eb_route_experts.argtypes = [i64, i32, i32, p, i32, i64, p, i32, i32, i32, ctypes.c_float, i32, i32, p, p, p, p, p,
                                         p, size, p]
        lib.eb_route_experts.restype = ctypes.c_int
        lib.eb_quantize_fp8.argtypes = [i32, i64, i64, p, i32, i64, i32, p, i64, p, i64, p]
        lib.eb_quantize_fp8.restype = ctypes.c_int
        lib.eb_expert_product.argtypes = [i64, i32, i64, i64, p, i64, i64, p, i64, p, p, i64, p, p, p, i32, i32, p, i64, p, i64, p]
        lib.eb_expert_product.restype = ctypes.c_int
        _lib = lib
    return _lib


def eb_route_experts_workspace(N: int, K: int, shard_lo: int, shard_hi: int) -> int:
    n = ctypes.c_size_t()
    _check(library().eb_route_experts_workspace(N, K, shard_lo, shard_hi, ctypes.byref(n)))
    return n.value


def eb_route_experts(N: int, E: int, K: int, scores_ptr: int | None, dtype: int, ld: int, bias_ptr: int | None, mode: int,
                     groups: int, top_groups: int, scale: float, shard_lo: int, shard_hi: int, ids_ptr: int | None,
                     weights_ptr: int | None, offsets_ptr: int | None, tokens_ptr: int | None, slots_ptr: int | None,
                     workspace_ptr: int | None, workspace_bytes: int, stream_ptr: int | None) -> None:
    """Enqueue the routing on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_route_experts(N, E, K, scores_ptr or None, dtype, ld, bias_ptr or None, mode, groups, top_groups,
                                      scale, shard_lo, shard_hi, ids_ptr or None, weights_ptr or None, offsets_ptr or None,
                                      tokens_ptr or None, slots_ptr or None, workspace_ptr or None, workspace_bytes,
                                      stream_ptr or None))


def eb_quantize_fp8(matrices: int, rows: int, cols: int, x_ptr: int | None, dtype: int, ldx: int, block_rows: int,
                    q_ptr: int | None, ldq: int, scales_ptr: int | None, lds: int, stream_ptr: int | None) -> None:
    """Enqueue the quantisation on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_quantize_fp8(matrices, rows, cols, x_ptr or None, dtype, ldx, block_rows, q_ptr or None, ldq,
                                     scales_ptr or None, lds, stream_ptr or None))


def eb_expert_product(M: int, E: int, N: int, K: int, x_ptr: int | None, ldx: int, x_rows: int, x_scales_ptr: int | None,
                      ldxs: int, tokens_ptr: int | None, w_ptr: int | None, ldw: int, w_scales_ptr: int | None,
                      offsets_ptr: int | None, bias_ptr: int | None, act: int, out_type: int, out_ptr: int | None,
                      ldo: int, out_scales_ptr: int | None, ldos: int, stream_ptr: int | None) -> None:
    """Enqueue the product on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_expert_product(M, E, N, K, x_ptr or None, ldx, x_rows, x_scales_ptr or None, ldxs, tokens_ptr or None,
                                       w_ptr or None, ldw, w_scales_ptr or None, offsets_ptr or None, bias_ptr or None, act,
                                       out_type, out_ptr or None, ldo, out_scales_ptr or None, ldos, stream_ptr or None))


_codes = {}


def _code(dtype, fp8: bool = False) -> int:
    if not _codes:
        import torch

        _codes.update({torch.float32: EB_F32, torch.float16: EB_F16, torch.bfloat16: EB_BF16, torch.float8_e4m3fn: EB_FP8})
    code = _codes.get(dtype)
    if code is None or (code == EB_FP8 and not fp8):
        raise ValueError(f"unsupported dtype {dtype}")
    return code


def _maker(x, stream):
    """empty(shape, dtype) on x's device, from ``stream``'s memory where one is
    given: what the caching allocator hands out again is then ordered with it."""
    import torch

    if stream is None:
        return lambda shape, dtype: x.new_empty(shape, dtype=dtype)

    def empty(shape, dtype):
        with torch.cuda.stream(stream):
            return x.new_empty(shape, dtype=dtype)

    return empty


def _blocks(n: int) -> int:
    return -(-n // BLOCK)


def _pitch(t, what: str) -> int:
    """Elements between the rows of a 2-D tensor of unit column stride."""
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} must have unit column stride")
    ld = t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])
    if ld < t.shape[1]:
        raise ValueError(f"{what} must have rows that do not overlap")
    return ld


class Route(NamedTuple):
    """What ``route`` returns; see eb_route_experts."""
    ids: object      # int32 [N, K]
    weights: object  # fp32 [N, K]
    offsets: object  # int32 [shard_hi - shard_lo + 1], or None
    tokens: object   # int32 [N * K], or None
    slots: object    # int32 [N, K], or None


def route(scores, top: int, mode: int = EB_SOFTMAX | EB_RENORMALIZE, bias=None, groups: int = 1, top_groups: int = 1,
          scale: float = 1.0, shard_lo: int = 0, shard_hi: int | None = None, grouped: bool = True, stream=None) -> Route:
    """Torch convenience for eb_route_experts.  ``scores``: device [N, E] of
    fp32, fp16 or bf16 with unit column stride; ``bias``: contiguous fp32 [E]
    or None.  ``grouped=False`` gives ids and weights only."""
    import torch

    if scores.dim() != 2 or not scores.is_cuda:
        raise ValueError("scores must be a 2-D device tensor")
    N, E = scores.shape
    dtype, ld, dev = _code(scores.dtype), _pitch(scores, "scores"), scores.device
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_contiguous() or bias.numel() != E):
        raise ValueError("bias must be contiguous fp32 [E]")
    _same_device(dev, bias)
    hi = E if shard_hi is None else int(shard_hi)
    empty = _maker(scores, stream)
    ids = empty((N, top), torch.int32)
    weights = empty((N, top), torch.float32)
    offsets = tokens = slots = ws = None
    nbytes = 0
    if grouped:
        nbytes = eb_route_experts_workspace(N, top, shard_lo, hi)
        offsets = empty((hi - shard_lo + 1,), torch.int32)
        tokens = empty((N * top,), torch.int32)
        slots = empty((N, top), torch.int32)
        ws = empty((nbytes,), torch.uint8)
    _check(library().eb_route_experts(
        N, E, top, scores.data_ptr() or None, dtype, ld, bias.data_ptr() if bias is not None else None, mode, groups,
        top_groups, scale, shard_lo, hi, ids.data_ptr() or None, weights.data_ptr() or None,
        offsets.data_ptr() if grouped else None, (tokens.data_ptr() or None) if grouped else None,
        (slots.data_ptr() or None) if grouped else None, ws.data_ptr() if grouped else None, nbytes,
        _stream_ptr(stream, dev) or None))
    return Route(ids, weights, offsets, tokens, slots)


def quantize_fp8(x, block_rows: int = 1, stream=None):
    """Torch convenience for eb_quantize_fp8.  ``x``: device [rows, cols] or
    [matrices, rows, cols] of fp32, fp16 or bf16 with unit column stride,
    matrices stacked row after row.  Returns (q, scales): q float8_e4m3fn of
    x's shape (its rows a multiple of 16 bytes apart); scales fp32
    [.., blocks of rows, ceil(cols/128)], for ``block_rows`` 1 with the scales
    of one column of blocks side by side in memory."""
    import torch

    if x.dim() not in (2, 3) or not x.is_cuda:
        raise ValueError("x must be a 2-D or 3-D device tensor")
    m, (rows, cols) = (x.shape[0] if x.dim() == 3 else 1), x.shape[-2:]
    flat = x if x.dim() == 2 else (x[0] if m else x.reshape(0, cols))
    dtype, ldx = _code(x.dtype), _pitch(flat, "x")
    if m > 1 and rows == 1:
        ldx = x.stride(0)
    elif m > 1 and x.stride(0) != rows * ldx:
        raise ValueError("x's matrices must be stacked row after row")
    empty = _maker(x, stream)
    pitch = -(-cols // 16) * 16
    q = empty((m, rows, pitch), torch.float8_e4m3fn)[:, :, :cols]
    if block_rows == 1:
        scales = empty((_blocks(cols), m * rows), torch.float32)
        lds, shaped = m * rows, scales.t()
        shaped = shaped.view(m, rows, -1) if x.dim() == 3 else shaped
    else:
        scales = empty((m, _blocks(rows), _blocks(cols)), torch.float32)
        lds, shaped = 0, scales if x.dim() == 3 else scales[0]
    _check(library().eb_quantize_fp8(m, rows, cols, x.data_ptr() or None, dtype, ldx, block_rows, q.data_ptr() or None, pitch,
                                     scales.data_ptr() or None, lds, _stream_ptr(stream, x.device) or None))
    return (q if x.dim() == 3 else q[0]), shaped


def product(x, x_scales, w, w_scales, offsets=None, tokens=None, bias=None, act: int = EB_ACT_NONE, out_dtype=None,
            out=None, stream=None):
    """Torch convenience for eb_expert_product.  ``x``: float8_e4m3fn [rows, K]
    and ``x_scales`` fp32 [rows, ceil(K/128)] as ``quantize_fp8`` gives them;
    ``w``: float8_e4m3fn [N, K] or [E, N, K] and ``w_scales`` as
    ``quantize_fp8(.., block_rows=128)`` gives them (under EB_ACT_SILU_GATE
    with the halves of N blocked each on its own: [E, 2 * ceil(N/2/128),
    ceil(K/128)]).  ``offsets``: int32 [E + 1] and ``tokens``: int32 [slots], or
    None, as ``route`` gives them; ``bias``: fp32 [N] or [E, N].  Returns the
    output [slots, width] of ``out_dtype`` (bfloat16), or for float8_e4m3fn
    (output, scales [slots, ceil(width/128)]).  Slots of no expert are not
    written.  ``out``: the floating-point output, with unit column stride."""
    import torch

    if x.dim() != 2 or w.dim() not in (2, 3) or not x.is_cuda:
        raise ValueError("x must be a 2-D device tensor, w 2-D or 3-D")
    if x.dtype != torch.float8_e4m3fn or w.dtype != torch.float8_e4m3fn:
        raise ValueError("x and w must be float8_e4m3fn")
    dev, (rows, K), (N, wk) = x.device, x.shape, w.shape[-2:]
    E = w.shape[0] if w.dim() == 3 else 1
    if wk != K or E == 0:
        raise ValueError("w must be [N, K] or [E, N, K], E at least 1")
    ldw = _pitch(w if w.dim() == 2 else w[0], "w")
    if E > 1 and N == 1:
        ldw = w.stride(0)
    elif E > 1 and w.stride(0) != N * ldw:
        raise ValueError("w's matrices must be stacked row after row")
    ldx, kb = _pitch(x, "x"), _blocks(K)
    gate = act == EB_ACT_SILU_GATE
    width = N // 2 if gate else N
    if x_scales.dtype != torch.float32 or tuple(x_scales.shape) != (rows, kb):
        raise ValueError("x_scales must be fp32 [rows, ceil(K/128)]")
    if rows > 1 and x_scales.stride(0) != 1 or kb > 1 and x_scales.stride(1) < rows:
        x_scales = x_scales.t().contiguous().t()
    ldxs = x_scales.stride(1) if kb > 1 else rows
    if w_scales.dtype != torch.float32 or not w_scales.is_contiguous() or \
            w_scales.numel() != E * (2 if gate else 1) * _blocks(width) * kb:
        raise ValueError("w_scales must be contiguous fp32, a scale per 128 x 128 of w")
    if offsets is not None and (offsets.dtype != torch.int32 or not offsets.is_contiguous() or offsets.numel() != E + 1):
        raise ValueError("offsets must be contiguous int32 [E + 1]")
    if tokens is not None and (tokens.dtype != torch.int32 or not tokens.is_contiguous()):
        raise ValueError("tokens must be contiguous int32")
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_contiguous() or bias.numel() != E * N):
        raise ValueError("bias must be contiguous fp32 [E, N]")
    _same_device(dev, x_scales, w, w_scales, offsets, tokens, bias, out)
    M = rows if tokens is None else tokens.numel()
    out_dtype = out.dtype if out is not None else torch.bfloat16 if out_dtype is None else out_dtype
    code = _code(out_dtype, fp8=True)
    empty, scales = _maker(x, stream), None
    if code == EB_FP8:
        if out is not None:
            raise ValueError("out is for floating-point outputs")
        ldo = -(-width // 16) * 16
        out = empty((M, ldo), out_dtype)[:, :width]
        scales = empty((_blocks(width), M), torch.float32)
    else:
        if out is None:
            out = empty((M, width), out_dtype)
        elif tuple(out.shape) != (M, width):
            raise ValueError("out must be [slots, width]")
        ldo = _pitch(out, "out")
    _check(library().eb_expert_product(
        M, E, N, K, x.data_ptr() or None, ldx, rows, x_scales.data_ptr() or None, ldxs,
        (tokens.data_ptr() or None) if tokens is not None else None, w.data_ptr() or None, ldw, w_scales.data_ptr() or None,
        offsets.data_ptr() if offsets is not None else None, bias.data_ptr() if bias is not None else None, act, code,
        out.data_ptr() or None, ldo, scales.data_ptr() or None if scales is not None else None, M,
        _stream_ptr(stream, dev) or None))
    return (out, scales.t()) if code == EB_FP8 else out
