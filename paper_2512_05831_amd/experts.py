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

import contextlib
import ctypes
import functools
from typing import NamedTuple

from . import eb
from .eb import EB_BF16, EB_F16, EB_F32, EB_SUM, _check

EB_FP8 = 3
EB_SOFTMAX, EB_SIGMOID = 0, 1
EB_RENORMALIZE, EB_GROUP_PAIR = 0x100, 0x200
EB_ACT_NONE, EB_ACT_RELU, EB_ACT_SILU_GATE = 0, 1, 2
EB_EXACT_SUMS = 0x100
BLOCK = 128

_lib = None


def library() -> ctypes.CDLL:
    """``eb.library()`` with the experts' functions declared."""
    global _lib
    if _lib is None:
        lib = eb.library()
        p, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        lib.eb_route_experts_workspace.argtypes = [i64, i32, i32, i32, i32, ctypes.POINTER(size)]
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


def eb_route_experts_workspace(N: int, E: int, K: int, shard_lo: int, shard_hi: int) -> int:
    n = ctypes.c_size_t()
    _check(library().eb_route_experts_workspace(N, E, K, shard_lo, shard_hi, ctypes.byref(n)))
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


def _gpu() -> int:
    """The current GPU's number; from the second call on torch's own query itself
    (0.06 us against current_device's 0.25)."""
    global _gpu
    import torch

    _gpu = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _gpu()


def _raw_stream(index: int) -> int:
    """The hipStream_t of GPU ``index``'s current stream; from the second call on
    torch's own query itself, where it offers one."""
    global _raw_stream
    import torch

    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(index)


def _place(torch, x, stream):
    """Where a call on ``x`` belongs, as a context.  Under a ``stream``
    allocations are the stream's: what the caching allocator hands out again is
    then ordered with it.  Else it is the GPU of ``x``: kernels on a default
    stream run on the current one.  (Callers ask only where that is not so
    already: a context takes longer than the rest of a call's checks.)"""
    if stream is not None:
        return torch.cuda.stream(stream)
    return torch.cuda.device(x.device) if x.is_cuda else contextlib.nullcontext()


def _same_device(dev, *tensors) -> None:
    """Every tensor given (None skipped) lives on the GPU ``dev``."""
    index = dev.index
    for x in tensors:
        if x is not None and x.get_device() != index:
            raise ValueError(f"tensor on {x.device}, expected {dev}")


def _blocks(n: int) -> int:
    return -(-n // BLOCK)


def _pitch(t, what: str) -> int:
    """Elements between the rows of a 2-D tensor of unit column stride."""
    (rows, cols), (ld, unit) = t.shape, t.stride()
    if unit != 1 and cols > 1:
        raise ValueError(f"{what} must have unit column stride")
    if ld < cols:
        if rows > 1:
            raise ValueError(f"{what} must have rows that do not overlap")
        return cols
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
    or None.  ``grouped=False`` gives ids and weights only.  The results share
    one allocation."""
    import torch

    if stream is None and -1 < scores.get_device() == _gpu():
        return _route(torch, scores, top, mode, bias, groups, top_groups, scale, shard_lo, shard_hi, grouped, None)
    with _place(torch, scores, stream):
        return _route(torch, scores, top, mode, bias, groups, top_groups, scale, shard_lo, shard_hi, grouped, stream)


def _route(torch, scores, top, mode, bias, groups, top_groups, scale, lo, hi, grouped, stream):
    if scores.dim() != 2 or not scores.is_cuda:
        raise ValueError("scores must be a 2-D device tensor")
    N, E = scores.shape
    dtype, ld, dev, bias_ptr = _code(scores.dtype), _pitch(scores, "scores"), scores.device, None
    if bias is not None:
        if bias.dtype != torch.float32 or not bias.is_contiguous() or bias.numel() != E:
            raise ValueError("bias must be contiguous fp32 [E]")
        _same_device(dev, bias)
        bias_ptr = bias.data_ptr()
    hi = E if hi is None else int(hi)
    lib = _lib or library()
    nbytes = _route_workspace(N, E, top, lo, hi) if grouped else 0
    if grouped:  # one allocation, 1.2 us less than five
        pairs = N * top
        whole = scores.new_empty((4 * pairs + hi - lo + 1,), dtype=torch.int32)
        each, tokens, offsets = whole.split_with_sizes((3 * pairs, pairs, hi - lo + 1))
        ids, slots, weights = each.view(3, N, top).unbind(0)
        weights = weights.view(torch.float32)
        ws = whole.new_empty((nbytes // 4,)) if nbytes else None
    else:
        ids = scores.new_empty((N, top), dtype=torch.int32)
        weights = torch.empty_like(ids, dtype=torch.float32)
        offsets = tokens = slots = ws = None
    rc = lib.eb_route_experts(
        N, E, top, scores.data_ptr(), dtype, ld, bias_ptr, mode, groups, top_groups, scale, lo, hi, ids.data_ptr(),
        weights.data_ptr(), offsets.data_ptr() if grouped else None, tokens.data_ptr() if grouped else None,
        slots.data_ptr() if grouped else None, ws.data_ptr() if nbytes else None, nbytes, _raw_stream(dev.index) if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)
    return Route(ids, weights, offsets, tokens, slots)


@functools.lru_cache(maxsize=256)
def _route_workspace(N, E, top, lo, hi):
    return eb_route_experts_workspace(N, E, top, lo, hi)


def quantize_fp8(x, block_rows: int = 1, stream=None):
    """Torch convenience for eb_quantize_fp8.  ``x``: device [rows, cols] or
    [matrices, rows, cols] of fp32, fp16 or bf16 with unit column stride,
    matrices stacked row after row.  Returns (q, scales): q float8_e4m3fn of
    x's shape (its rows a multiple of 16 bytes apart); scales fp32
    [.., blocks of rows, ceil(cols/128)], for ``block_rows`` 1 with the scales
    of one column of blocks side by side in memory."""
    import torch

    if stream is None and -1 < x.get_device() == _gpu():
        return _quantize(torch, x, block_rows, None)
    with _place(torch, x, stream):
        return _quantize(torch, x, block_rows, stream)


def _quantize(torch, x, block_rows, stream):
    dim = x.dim()
    if dim not in (2, 3) or not x.is_cuda:
        raise ValueError("x must be a 2-D or 3-D device tensor")
    if dim == 2:
        (rows, cols), m, ldx = x.shape, 1, _pitch(x, "x")
    else:
        m, rows, cols = x.shape
        ldx = _pitch(x[0], "x") if m else cols
        if m > 1 and rows == 1:
            ldx = x.stride(0)
        elif m > 1 and rows > 1 and x.stride(0) != rows * ldx:
            raise ValueError("x's matrices must be stacked row after row")
    dtype, pitch, blocks = _code(x.dtype), (cols + 15) & -16, (cols + BLOCK - 1) // BLOCK
    q = x.new_empty((rows, pitch) if dim == 2 else (m, rows, pitch), dtype=torch.float8_e4m3fn)
    if block_rows == 1:
        lds = m * rows
        if dim == 2:
            scales = shaped = x.new_empty_strided((rows, blocks), (1, lds), dtype=torch.float32)
        else:
            scales = shaped = x.new_empty_strided((m, rows, blocks), (rows, 1, lds), dtype=torch.float32)
    else:
        scales = x.new_empty((m, _blocks(rows), blocks), dtype=torch.float32)
        lds, shaped = 0, scales if dim == 3 else scales[0]
    rc = (_lib or library()).eb_quantize_fp8(m, rows, cols, x.data_ptr(), dtype, ldx, block_rows, q.data_ptr(), pitch,
                                             scales.data_ptr(), lds, _raw_stream(x.get_device()) if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)
    return (q if pitch == cols else q[..., :cols]), shaped


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
    written.  ``out``: the floating-point output, with unit column stride.
    ``act`` | EB_EXACT_SUMS: 16-bit outputs too from sums exact to fp32's
    rounding."""
    import torch

    if stream is None and -1 < x.get_device() == _gpu():
        return _product(torch, x, x_scales, w, w_scales, offsets, tokens, bias, act, out_dtype, out, None)
    with _place(torch, x, stream):
        return _product(torch, x, x_scales, w, w_scales, offsets, tokens, bias, act, out_dtype, out, stream)


def _product(torch, x, x_scales, w, w_scales, offsets, tokens, bias, act, out_dtype, out, stream):
    f8, f32, i32 = torch.float8_e4m3fn, torch.float32, torch.int32
    if x.dim() != 2 or w.dim() not in (2, 3) or not x.is_cuda:
        raise ValueError("x must be a 2-D device tensor, w 2-D or 3-D")
    if x.dtype != f8 or w.dtype != f8:
        raise ValueError("x and w must be float8_e4m3fn")
    dev, (rows, K) = x.device, x.shape
    if w.dim() == 2:
        (N, wk), E, ldw = w.shape, 1, _pitch(w, "w")
    else:
        E, N, wk = w.shape
        if E == 0:
            raise ValueError("w must hold an expert")
        ldw = _pitch(w[0], "w")
        if E > 1 and N == 1:
            ldw = w.stride(0)
        elif E > 1 and w.stride(0) != N * ldw:
            raise ValueError("w's matrices must be stacked row after row")
    if wk != K:
        raise ValueError("w must be [N, K] or [E, N, K]")
    ldx, kb = _pitch(x, "x"), (K + BLOCK - 1) // BLOCK
    gate = act & ~EB_EXACT_SUMS == EB_ACT_SILU_GATE
    width = N // 2 if gate else N
    blocks = (width + BLOCK - 1) // BLOCK
    if x_scales.dtype != f32 or x_scales.shape != (rows, kb):
        raise ValueError("x_scales must be fp32 [rows, ceil(K/128)]")
    by_row, by_block = x_scales.stride()
    if rows > 1 and by_row != 1 or kb > 1 and by_block < rows:
        x_scales = x_scales.t().contiguous().t()
        by_block = rows
    ldxs = by_block if kb > 1 else rows
    lines = 2 * blocks if gate else blocks
    if w_scales.dtype != f32 or not w_scales.is_contiguous() or w_scales.shape != ((lines, kb) if w.dim() == 2 else (E, lines, kb)) and (
            w_scales.numel() != E * lines * kb or w_scales.shape[-1:] != (kb,) or w_scales.shape[-2:-1] not in ((lines,), (blocks,))):
        raise ValueError("w_scales must be contiguous fp32 [.., blocks of N, ceil(K/128)], a scale per 128 x 128 of w")
    M, offsets_ptr, tokens_ptr, bias_ptr = rows, None, None, None
    if offsets is not None:
        if offsets.dtype != i32 or not offsets.is_contiguous() or offsets.numel() != E + 1:
            raise ValueError("offsets must be contiguous int32 [E + 1]")
        offsets_ptr = offsets.data_ptr()
    if tokens is not None:
        if tokens.dtype != i32 or not tokens.is_contiguous():
            raise ValueError("tokens must be contiguous int32")
        M, tokens_ptr = tokens.numel(), tokens.data_ptr()
    if bias is not None:
        if bias.dtype != f32 or not bias.is_contiguous() or bias.shape != (E, N) and (E > 1 or bias.shape != (N,)):
            raise ValueError("bias must be contiguous fp32 [E, N], or [N] of one expert")
        bias_ptr = bias.data_ptr()
    _same_device(dev, x_scales, w, w_scales, offsets, tokens, bias, out)
    scales_ptr, scales = None, None
    if out is not None and out_dtype is not None and out_dtype != out.dtype:
        raise ValueError("out is of another type than out_dtype")
    code = _code(out.dtype if out is not None else torch.bfloat16 if out_dtype is None else out_dtype, fp8=True)
    if code == EB_FP8:
        if out is not None:
            raise ValueError("out is for floating-point outputs")
        ldo = (width + 15) & -16
        out = x.new_empty((M, ldo))
        scales = x.new_empty_strided((M, blocks), (1, M), dtype=f32)
        scales_ptr = scales.data_ptr()
    elif out is None:
        ldo = width
        out = x.new_empty((M, width), dtype=torch.bfloat16 if out_dtype is None else out_dtype)
    else:
        if out.shape != (M, width):
            raise ValueError("out must be [slots, width]")
        ldo = _pitch(out, "out")
    rc = (_lib or library()).eb_expert_product(
        M, E, N, K, x.data_ptr(), ldx, rows, x_scales.data_ptr(), ldxs, tokens_ptr, w.data_ptr(), ldw, w_scales.data_ptr(),
        offsets_ptr, bias_ptr, act, code, out.data_ptr(), ldo, scales_ptr, M, _raw_stream(dev.index) if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)
    if code == EB_FP8:
        return (out if ldo == width else out[:, :width]), scales
    return out


class ExpertLayer:
    """A mixture of experts for inference: each token's ``top`` experts' two
    layers, joined with the router's weights.

    ``w_up``: [E, N, K] and ``w_down``: [E, D, N] (or, gated, [E, D, N / 2]) device
    tensors of fp32, fp16 or bf16, held here in 8 bits with a scale per
    128 x 128; ``router``: [experts, K] fp32, whose rows give the scores of all
    experts.  Row-wise over several GPUs, a GPU holds the experts
    [shard_lo, shard_lo + E) of them, as a row shard of a table holds rows: its
    results are partial sums, to be added over the GPUs (``sum_partials``).

    ``row_dtype``: the type in which the experts' rows wait to be joined, fp32,
    fp16 or bf16 (the default: one rounding to 8 bits of mantissa, beside hidden
    values that have 4; half of fp32's bytes, and the 8-bit matrix unit for the
    second product: 16384 tokens, 4 of 32 experts of 1024 x 512, 393 us, in fp32
    417).  The joined sums are fp32.  ``act`` | EB_EXACT_SUMS holds
    for both products."""

    def __init__(self, w_up, w_down, router, top: int, act: int = EB_ACT_SILU_GATE, mode: int = EB_SOFTMAX | EB_RENORMALIZE,
                 bias=None, groups: int = 1, top_groups: int = 1, scale: float = 1.0, shard_lo: int = 0, row_dtype=None):
        import torch

        if w_up.dim() != 3 or w_down.dim() != 3 or router.dim() != 2:
            raise ValueError("w_up and w_down must be 3-D, router 2-D")
        E, N, K = w_up.shape
        gate = act & ~EB_EXACT_SUMS == EB_ACT_SILU_GATE
        if gate and N % 2 or tuple(w_down.shape[::2]) != (E, N // 2 if gate else N) or router.shape[1] != K:
            raise ValueError("w_up [E, N, K], w_down [E, D, N or N / 2] and router [experts, K] do not fit")
        self.E, self.K, self.D, self.top, self.act, self.mode = E, K, int(w_down.shape[1]), top, act, mode
        self.router, self.bias, self.groups, self.top_groups, self.scale = router, bias, groups, top_groups, scale
        self.shard_lo = shard_lo
        self.row_dtype = torch.bfloat16 if row_dtype is None else row_dtype
        _code(self.row_dtype)
        # Under a gate each half of the rows is blocked on its own.
        parts = 2 if gate else 1
        q, s = quantize_fp8(w_up.contiguous().view(E * parts, N // parts, K), block_rows=BLOCK)
        self.w_up, self.up_scales = q.as_strided((E, N, K), (N * q.stride(1), q.stride(1), 1)), s.view(E, -1, s.shape[2])
        self.w_down, self.down_scales = quantize_fp8(w_down.contiguous(), block_rows=BLOCK)

    def forward(self, x, scores=None, out=None):
        """``x``: device [B, K] of fp32, fp16 or bf16, for example a batch's
        pooled lookups; ``scores``: [B, experts], or None for the router's.
        Returns fp32 [B, D]."""
        import torch

        if -1 < x.get_device() == _gpu():
            return self._forward(torch, x, scores, out)
        with _place(torch, x, None):
            return self._forward(torch, x, scores, out)

    def _forward(self, torch, x, scores, out):
        if x.dim() != 2 or x.shape[1] != self.K:
            raise ValueError("x must be [B, K]")
        B = int(x.shape[0])
        if scores is None:
            scores = x.float() @ self.router.t()
        elif scores.shape != (B, self.router.shape[0]):
            raise ValueError("scores must be [B, experts]")
        r = route(scores, self.top, self.mode, self.bias, self.groups, self.top_groups, self.scale, self.shard_lo,
                  self.shard_lo + self.E)
        q, s = quantize_fp8(x)
        h, hs = product(q, s, self.w_up, self.up_scales, r.offsets, r.tokens, act=self.act, out_dtype=torch.float8_e4m3fn)
        y = product(h, hs, self.w_down, self.down_scales, r.offsets, act=self.act & EB_EXACT_SUMS, out_dtype=self.row_dtype)
        bags = torch.arange(0, B * self.top + 1, self.top, dtype=torch.int32, device=x.device)
        # A token is a bag of its pairs' slots; a pair without one (-1) is skipped.
        slots = eb.EmbeddingBagTables([y])
        out = slots.forward_ex(r.slots.view(-1), bags, B, EB_SUM, out=out, weights=r.weights.view(-1))
        slots.close()
        return out
