"""Python binding of the C ABI in ``include/eb_train.h`` (ctypes, marshalling only).

What trains a mixture of experts over pooled lookups, beside ``experts``:
``layer_norm`` and ``layer_norm_backward``, ``activation`` and
``activation_backward`` of values that wait in 8 bits, ``dispatch``, ``combine`` and
``combine_backward`` (rows sorted by expert and joined again), ``weight_gradient``.
``eb_layer_norm`` and its like are the C calls under their own names, with device
addresses as ints.  There is no fallback: every step runs in ``libeb.so``.

A matrix in 8 bits is a pair (values, scales) as ``experts.quantize_fp8`` returns it
with a scale per 1 x 128.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import math
from typing import NamedTuple

import torch

from . import eb, experts as ex
from .eb import EB_BF16, EB_F16, EB_F32, _check
from .experts import BLOCK, EB_ACT_SILU_GATE, EB_FP8, _place

_lib = None


def library() -> ctypes.CDLL:
    """``eb.library()`` with the functions of eb_train.h declared."""
    global _lib
    if _lib is None:
        lib = eb.library()
        p, i32, i64, size, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        for name, args in (
                ("eb_layer_norm", [i64, i64, p, i32, i64, p, p, f32, i32, p, i64, p, i64, p, i64, p, i64, p, p, p]),
                ("eb_layer_norm_backward_workspace", [i64, i64, ctypes.POINTER(size)]),
                ("eb_layer_norm_backward", [i64, i64, p, i32, i64, p, i32, i64, p, i64, p, p, p, p, i64, p, p, p, size, p]),
                ("eb_activation", [i64, i64, i32, p, i32, i64, p, i64, i32, p, i64, p, i64, p]),
                ("eb_activation_backward", [i64, i64, i32, p, i32, i64, p, i32, i64, p, i64, i32, p, i64, p, i64, p]),
                ("eb_dispatch", [i64, i64, p, i32, i64, i64, p, i64, p, p, i64, p, i64, p]),
                ("eb_combine", [i64, i32, i64, p, i32, i64, i64, p, p, i32, p, i64, p]),
                ("eb_combine_backward", [i64, i32, i64, p, i32, i64, p, i32, i64, i64, p, p, i32, p, i64, p, i64, p, p]),
                ("eb_weight_gradient_workspace", [i64, i32, i64, i64, ctypes.POINTER(size)]),
                ("eb_weight_gradient", [i64, i32, i64, i64, p, i32, i64, p, i64, p, i32, i64, i64, p, i64, p, p, i32, i32, p, i64, p, size, p])):
            f = getattr(lib, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _lib = lib
    return _lib


def eb_layer_norm(rows: int, cols: int, x_ptr: int | None, dtype: int, ldx: int, weight_ptr: int | None, bias_ptr: int | None, eps: float,
                  out_type: int, y_ptr: int | None, ldy: int, y_scales_ptr: int | None, ldys: int, kept_ptr: int | None, ldk: int,
                  kept_scales_ptr: int | None, ldks: int, mean_ptr: int | None, rstd_ptr: int | None, stream_ptr: int | None) -> None:
    """Enqueue the layer norm on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_layer_norm(rows, cols, x_ptr or None, dtype, ldx, weight_ptr or None, bias_ptr or None, eps, out_type, y_ptr or None,
                                   ldy, y_scales_ptr or None, ldys, kept_ptr or None, ldk, kept_scales_ptr or None, ldks, mean_ptr or None,
                                   rstd_ptr or None, stream_ptr or None))


def eb_layer_norm_backward_workspace(rows: int, cols: int) -> int:
    n = ctypes.c_size_t()
    _check(library().eb_layer_norm_backward_workspace(rows, cols, ctypes.byref(n)))
    return n.value


def eb_layer_norm_backward(rows: int, cols: int, dy_ptr: int | None, dy_type: int, lddy: int, x_ptr: int | None, x_type: int, ldx: int,
                           x_scales_ptr: int | None, ldxs: int, mean_ptr: int | None, rstd_ptr: int | None, weight_ptr: int | None,
                           dx_ptr: int | None, lddx: int, dweight_ptr: int | None, dbias_ptr: int | None, workspace_ptr: int | None,
                           workspace_bytes: int, stream_ptr: int | None) -> None:
    """Enqueue the layer norm's gradients on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_layer_norm_backward(rows, cols, dy_ptr or None, dy_type, lddy, x_ptr or None, x_type, ldx, x_scales_ptr or None, ldxs,
                                            mean_ptr or None, rstd_ptr or None, weight_ptr or None, dx_ptr or None, lddx, dweight_ptr or None,
                                            dbias_ptr or None, workspace_ptr or None, workspace_bytes, stream_ptr or None))


def eb_activation(rows: int, cols: int, act: int, v_ptr: int | None, v_type: int, ldv: int, v_scales_ptr: int | None, ldvs: int, out_type: int,
                  h_ptr: int | None, ldh: int, h_scales_ptr: int | None, ldhs: int, stream_ptr: int | None) -> None:
    """Enqueue the activation on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_activation(rows, cols, act, v_ptr or None, v_type, ldv, v_scales_ptr or None, ldvs, out_type, h_ptr or None, ldh,
                                   h_scales_ptr or None, ldhs, stream_ptr or None))


def eb_activation_backward(rows: int, cols: int, act: int, dh_ptr: int | None, dh_type: int, lddh: int, v_ptr: int | None, v_type: int,
                           ldv: int, v_scales_ptr: int | None, ldvs: int, out_type: int, dv_ptr: int | None, lddv: int,
                           dv_scales_ptr: int | None, lddvs: int, stream_ptr: int | None) -> None:
    """Enqueue the activation's gradient on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_activation_backward(rows, cols, act, dh_ptr or None, dh_type, lddh, v_ptr or None, v_type, ldv, v_scales_ptr or None,
                                            ldvs, out_type, dv_ptr or None, lddv, dv_scales_ptr or None, lddvs, stream_ptr or None))


def eb_dispatch(M: int, cols: int, x_ptr: int | None, dtype: int, ldx: int, x_rows: int, x_scales_ptr: int | None, ldxs: int,
                tokens_ptr: int | None, out_ptr: int | None, ldo: int, out_scales_ptr: int | None, ldos: int, stream_ptr: int | None) -> None:
    """Enqueue the sorting on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_dispatch(M, cols, x_ptr or None, dtype, ldx, x_rows, x_scales_ptr or None, ldxs, tokens_ptr or None, out_ptr or None,
                                 ldo, out_scales_ptr or None, ldos, stream_ptr or None))


def eb_combine(N: int, K: int, cols: int, y_ptr: int | None, y_type: int, ldy: int, y_rows: int, slots_ptr: int | None,
               weights_ptr: int | None, out_type: int, out_ptr: int | None, ldo: int, stream_ptr: int | None) -> None:
    """Enqueue the joining on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_combine(N, K, cols, y_ptr or None, y_type, ldy, y_rows, slots_ptr or None, weights_ptr or None, out_type,
                                out_ptr or None, ldo, stream_ptr or None))


def eb_combine_backward(N: int, K: int, cols: int, dout_ptr: int | None, dout_type: int, lddo: int, y_ptr: int | None, y_type: int, ldy: int,
                        y_rows: int, slots_ptr: int | None, weights_ptr: int | None, dy_type: int, dy_ptr: int | None, lddy: int,
                        dy_scales_ptr: int | None, lddys: int, dweights_ptr: int | None, stream_ptr: int | None) -> None:
    """Enqueue the joining's gradients on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_combine_backward(N, K, cols, dout_ptr or None, dout_type, lddo, y_ptr or None, y_type, ldy, y_rows, slots_ptr or None,
                                         weights_ptr or None, dy_type, dy_ptr or None, lddy, dy_scales_ptr or None, lddys,
                                         dweights_ptr or None, stream_ptr or None))


def eb_weight_gradient_workspace(M: int, E: int, N: int, K: int) -> int:
    n = ctypes.c_size_t()
    _check(library().eb_weight_gradient_workspace(M, E, N, K, ctypes.byref(n)))
    return n.value


def eb_weight_gradient(M: int, E: int, N: int, K: int, dy_ptr: int | None, dy_type: int, lddy: int, dy_scales_ptr: int | None, lddys: int,
                       x_ptr: int | None, x_type: int, ldx: int, x_rows: int, x_scales_ptr: int | None, ldxs: int, tokens_ptr: int | None,
                       offsets_ptr: int | None, out_type: int, accumulate: int, dw_ptr: int | None, lddw: int, workspace_ptr: int | None,
                       workspace_bytes: int, stream_ptr: int | None) -> None:
    """Enqueue the weights' gradients on ``stream_ptr``.  Raises EbError."""
    _check(library().eb_weight_gradient(M, E, N, K, dy_ptr or None, dy_type, lddy, dy_scales_ptr or None, lddys, x_ptr or None, x_type, ldx,
                                        x_rows, x_scales_ptr or None, ldxs, tokens_ptr or None, offsets_ptr or None, out_type, accumulate,
                                        dw_ptr or None, lddw, workspace_ptr or None, workspace_bytes, stream_ptr or None))


# --------------------------------------------------------------------------- torch


_F32, _I32, _BF16, _FP8 = torch.float32, torch.int32, torch.bfloat16, torch.float8_e4m3fn
_CODES = {_F32: EB_F32, torch.float16: EB_F16, _BF16: EB_BF16, _FP8: EB_FP8}


def _code(dtype) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise ValueError(f"unsupported dtype {dtype}")
    return code


def _placed(f):
    """The call under its ``stream``, or on its first tensor's GPU: at once where that is current."""
    first, last = f.__code__.co_varnames[0], f.__code__.co_argcount - 1  # the last one is the stream

    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        if len(args) == last + 1 and stream is None:
            args, stream = args[:last], args[last]
        x = args[0] if args else kw.get(first)
        if stream is None and x is not None and -1 < x.get_device() == ex._gpu():
            return f(*args, **kw)
        if x is None or not x.is_cuda:
            inspect.signature(f).bind(*args, **kw)
            raise ValueError("expected device tensors")
        with _place(torch, x, stream):
            return f(*args, stream=stream, **kw)
    return call


def _stream(x, stream):
    return ex._raw_stream(x.get_device()) if stream is None else stream.cuda_stream


def _floating(x, what: str):
    """(pointer, code, pitch) of a 2-D tensor of fp32, fp16 or bf16 with unit column stride."""
    code = _CODES.get(x.dtype)
    if code is None or code == EB_FP8 or x.dim() != 2:
        raise ValueError(f"{what} must be 2-D, fp32, fp16 or bf16")
    return x.data_ptr(), code, ex._pitch(x, what)


def _matrix(x, what: str, scales):
    """(pointer, code, pitch, scales' pointer, scales' pitch, the scales in use) of a 2-D
    tensor with unit column stride, in 8 bits with its scales."""
    code = _CODES.get(x.dtype)
    if code is None or x.dim() != 2:
        raise ValueError(f"{what} must be 2-D, fp32, fp16, bf16 or float8_e4m3fn")
    ld = ex._pitch(x, what)
    if code != EB_FP8:
        if scales is not None:
            raise ValueError(f"{what} is not in 8 bits: it takes no scales")
        return x.data_ptr(), code, ld, None, 0, None
    rows, n = x.shape
    blocks = (n + BLOCK - 1) // BLOCK
    if scales is None or scales.dtype != _F32 or scales.shape != (rows, blocks):
        raise ValueError(f"{what} in 8 bits needs its scales, fp32 [rows, ceil(columns/128)]")
    if scales.get_device() != x.get_device():
        raise ValueError(f"the scales of {what} are on {scales.device}, expected {x.device}")
    by_row, by_block = scales.stride()
    if rows > 1 and by_row != 1 or blocks > 1 and by_block < rows:
        scales = scales.t().contiguous().t()
        by_block = rows
    return x.data_ptr(), code, ld, scales.data_ptr(), by_block if blocks > 1 else rows, scales


def _new(like, rows: int, cols: int, dtype):
    """An output matrix beside ``like``: (tensor, code, pitch, scales or None, their pointer)."""
    code = _code(dtype)
    if code != EB_FP8:
        return like.new_empty((rows, cols), dtype=dtype), code, cols, None, None
    ld = cols + 15 & -16
    q = like.new_empty((rows, ld), dtype=dtype)
    scales = like.new_empty_strided((rows, (cols + BLOCK - 1) // BLOCK), (1, rows), dtype=_F32)
    return (q if ld == cols else q[:, :cols]), code, ld, scales, scales.data_ptr()


def _vector(x, what: str, dtype, dev, *shape):
    """The address of a contiguous tensor of a type and shape on a GPU; None of None."""
    if x is None:
        return None
    if x.dtype != dtype or x.shape != shape or not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} {list(shape)}")
    if x.get_device() != dev:
        raise ValueError(f"{what} is on {x.device}, expected GPU {dev}")
    return x.data_ptr()


class Norm(NamedTuple):
    """What ``layer_norm`` returns; see eb_layer_norm.  None what was not asked for."""
    y: object
    y_scales: object     # of a y in 8 bits
    mean: object         # fp32 [rows]
    rstd: object         # fp32 [rows]
    kept: object         # float8_e4m3fn [rows, cols]: the normalised values
    kept_scales: object


@_placed
def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out_dtype=None, statistics: bool = False, checkpoint: bool = False,
               stream=None) -> Norm:
    """Torch convenience for eb_layer_norm.  ``x``: device [rows, cols] of fp32, fp16 or
    bf16 with unit column stride; ``weight``, ``bias``: contiguous fp32 [cols] or None;
    ``out_dtype``: y's type (bfloat16), float8_e4m3fn for 8 bits with scales.  For the
    backward pass ``statistics`` gives mean and rstd (the caller keeps x), ``checkpoint``
    rstd and the normalised values in 8 bits."""
    ptr, code, ldx = _floating(x, "x")
    (rows, cols), dev = x.shape, x.get_device()
    y, out_type, ldy, y_scales, ys_ptr = _new(x, rows, cols, out_dtype or _BF16)
    mean = rstd = kept = kept_scales = None
    mean_ptr = rstd_ptr = kept_ptr = ks_ptr = None
    ldk = 0
    if statistics:
        mean, rstd = x.new_empty((2, rows), dtype=_F32).unbind(0)
        mean_ptr, rstd_ptr = mean.data_ptr(), rstd.data_ptr()
    elif checkpoint:
        rstd = x.new_empty((rows,), dtype=_F32)
        rstd_ptr = rstd.data_ptr()
    if checkpoint:
        kept, _, ldk, kept_scales, ks_ptr = _new(x, rows, cols, _FP8)
        kept_ptr = kept.data_ptr()
    rc = (_lib or library()).eb_layer_norm(
        rows, cols, ptr, code, ldx, _vector(weight, "weight", _F32, dev, cols), _vector(bias, "bias", _F32, dev, cols), eps, out_type,
        y.data_ptr(), ldy, ys_ptr, rows, kept_ptr, ldk, ks_ptr, rows, mean_ptr, rstd_ptr, _stream(x, stream))
    if rc:
        _check(rc)
    return Norm(y, y_scales, mean, rstd, kept, kept_scales)


@functools.lru_cache(maxsize=256)
def _norm_workspace(rows, cols):
    return eb_layer_norm_backward_workspace(rows, cols)


@_placed
def layer_norm_backward(dy, x, rstd, mean=None, x_scales=None, weight=None, parameters: bool = True, stream=None):
    """Torch convenience for eb_layer_norm_backward.  ``dy``: device [rows, cols] of fp32,
    fp16 or bf16; ``x`` with ``mean``: forward's input; or ``x`` (8 bits) with ``x_scales``:
    what it kept; ``weight``: forward's.  Returns (dx of dy's type, dweight, dbias), the
    last two fp32 [cols], or None without ``parameters``."""
    dy_ptr, dy_type, lddy = _floating(dy, "dy")
    (rows, cols), dev = dy.shape, dy.get_device()
    if x.shape != dy.shape or x.get_device() != dev:
        raise ValueError("x must have dy's shape, on its GPU")
    x_ptr, x_type, ldx, xs_ptr, ldxs, held = _matrix(x, "x", x_scales)
    if (x_type == EB_FP8) != (mean is None):
        raise ValueError("mean goes with an x in floating point, and only with that")
    dx = dy.new_empty((rows, cols))
    dweight = dbias = work = None
    dw_ptr = db_ptr = work_ptr = None
    nbytes = 0
    if parameters:
        nbytes = _norm_workspace(rows, cols)
        dweight, dbias = dy.new_empty((2, cols), dtype=_F32).unbind(0)
        work = dy.new_empty((nbytes // 4,), dtype=_F32)
        dw_ptr, db_ptr, work_ptr = dweight.data_ptr(), dbias.data_ptr(), work.data_ptr()
    rc = (_lib or library()).eb_layer_norm_backward(
        rows, cols, dy_ptr, dy_type, lddy, x_ptr, x_type, ldx, xs_ptr, ldxs, _vector(mean, "mean", _F32, dev, rows),
        _vector(rstd, "rstd", _F32, dev, rows), _vector(weight, "weight", _F32, dev, cols), dx.data_ptr(), cols, dw_ptr, db_ptr, work_ptr,
        nbytes, _stream(dy, stream))
    if rc:
        _check(rc)
    return dx, dweight, dbias


def _width_of_v(v, act):
    if v.dim() != 2 or (act == EB_ACT_SILU_GATE and v.shape[1] % 2):
        raise ValueError("v must be 2-D, under a gate with an even number of columns")
    return v.shape[1] // 2 if act == EB_ACT_SILU_GATE else v.shape[1]


@_placed
def activation(v, v_scales=None, act: int = EB_ACT_SILU_GATE, out_dtype=None, stream=None):
    """Torch convenience for eb_activation.  ``v``: device [rows, cols] (gated [rows, 2 *
    cols]) of fp32, fp16, bf16 or, with ``v_scales``, 8 bits.  Returns h [rows, cols] of
    ``out_dtype`` (bfloat16), or for float8_e4m3fn (h, scales)."""
    cols = _width_of_v(v, act)
    ptr, code, ldv, vs_ptr, ldvs, held = _matrix(v, "v", v_scales)
    rows = v.shape[0]
    h, out_type, ldh, scales, hs_ptr = _new(v, rows, cols, out_dtype or _BF16)
    rc = (_lib or library()).eb_activation(rows, cols, act, ptr, code, ldv, vs_ptr, ldvs, out_type, h.data_ptr(), ldh, hs_ptr, rows,
                                           _stream(v, stream))
    if rc:
        _check(rc)
    return h if scales is None else (h, scales)


@_placed
def activation_backward(dh, v, v_scales=None, act: int = EB_ACT_SILU_GATE, out_dtype=None, stream=None):
    """Torch convenience for eb_activation_backward.  ``dh``: device [rows, cols] of fp32,
    fp16 or bf16; ``v``, ``v_scales``, ``act``: forward's.  Returns dv, of v's shape and of
    ``out_dtype`` (bfloat16), or for float8_e4m3fn (dv, scales)."""
    cols = _width_of_v(v, act)
    dh_ptr, dh_type, lddh = _floating(dh, "dh")
    rows = dh.shape[0]
    if dh.shape[1] != cols or v.shape[0] != rows or v.get_device() != dh.get_device():
        raise ValueError("dh must be of h's shape, v on its GPU")
    ptr, code, ldv, vs_ptr, ldvs, held = _matrix(v, "v", v_scales)
    dv, out_type, lddv, scales, dvs_ptr = _new(dh, rows, v.shape[1], out_dtype or _BF16)
    rc = (_lib or library()).eb_activation_backward(rows, cols, act, dh_ptr, dh_type, lddh, ptr, code, ldv, vs_ptr, ldvs, out_type,
                                                    dv.data_ptr(), lddv, dvs_ptr, rows, _stream(dh, stream))
    if rc:
        _check(rc)
    return dv if scales is None else (dv, scales)


@_placed
def dispatch(x, tokens, x_scales=None, out=None, stream=None):
    """Torch convenience for eb_dispatch.  ``x``: device [rows, cols] of fp32, fp16, bf16 or,
    with ``x_scales``, 8 bits; ``tokens``: int32 [slots] as ``experts.route`` gives them.
    Returns [slots, cols] of x's type, in 8 bits (rows, scales); rows of slots without a
    token are not written.  ``out``: the floating-point output, with unit column stride."""
    ptr, code, ldx, xs_ptr, ldxs, held = _matrix(x, "x", x_scales)
    (rows, cols), M, dev = x.shape, tokens.numel(), x.get_device()
    tokens_ptr = _vector(tokens, "tokens", _I32, dev, M)
    scales = os_ptr = None
    if out is None:
        out, _, ldo, scales, os_ptr = _new(x, M, cols, x.dtype)
    else:
        if code == EB_FP8:
            raise ValueError("out is for floating-point rows")
        if out.dtype != x.dtype or out.shape != (M, cols) or out.get_device() != dev:
            raise ValueError("out must be [slots, cols] of x's type, on its GPU")
        ldo = ex._pitch(out, "out")
    rc = (_lib or library()).eb_dispatch(M, cols, ptr, code, ldx, rows, xs_ptr, ldxs, tokens_ptr, out.data_ptr(), ldo, os_ptr, M,
                                         _stream(x, stream))
    if rc:
        _check(rc)
    return out if scales is None else (out, scales)


@_placed
def combine(y, slots, weights=None, out_dtype=None, stream=None):
    """Torch convenience for eb_combine.  ``y``: device [rows, cols] of fp32, fp16 or bf16;
    ``slots``: int32 [tokens, K] as ``experts.route`` gives them; ``weights``: fp32
    [tokens, K] or None.  Returns [tokens, cols] of ``out_dtype`` (y's type)."""
    ptr, code, ldy = _floating(y, "y")
    if slots.dim() != 2:
        raise ValueError("slots must be 2-D")
    (rows, cols), (N, K), dev = y.shape, slots.shape, y.get_device()
    slots_ptr, weights_ptr = _vector(slots, "slots", _I32, dev, N, K), _vector(weights, "weights", _F32, dev, N, K)
    out_type = code if out_dtype is None else _code(out_dtype)
    if out_type == EB_FP8:
        raise ValueError("out_dtype must be fp32, fp16 or bf16")
    out = y.new_empty((N, cols), dtype=out_dtype or y.dtype)
    rc = (_lib or library()).eb_combine(N, K, cols, ptr, code, ldy, rows, slots_ptr, weights_ptr, out_type, out.data_ptr(), cols,
                                        _stream(y, stream))
    if rc:
        _check(rc)
    return out


class CombineGradient(NamedTuple):
    """What ``combine_backward`` returns; see eb_combine_backward."""
    dy: object
    dy_scales: object  # of a dy in 8 bits, else None
    dweights: object   # fp32 [tokens, K]


@_placed
def combine_backward(dout, y, slots, weights=None, out_dtype=None, stream=None) -> CombineGradient:
    """Torch convenience for eb_combine_backward.  ``dout``: device [tokens, cols] of fp32,
    fp16 or bf16; ``y``, ``slots``, ``weights``: forward's, no slot twice.  dy is of y's
    shape and ``out_dtype`` (y's type; float8_e4m3fn: 8 bits with scales); its rows that are
    no pair's slot are not written."""
    dout_ptr, dout_type, lddo = _floating(dout, "dout")
    ptr, code, ldy = _floating(y, "y")
    dev, (rows, cols) = dout.get_device(), y.shape
    if slots.dim() != 2 or dout.shape != (slots.shape[0], cols) or y.get_device() != dev:
        raise ValueError("dout must be [tokens, columns of y], slots [tokens, K], y on dout's GPU")
    N, K = slots.shape
    slots_ptr, weights_ptr = _vector(slots, "slots", _I32, dev, N, K), _vector(weights, "weights", _F32, dev, N, K)
    dy, dy_type, lddy, scales, dys_ptr = _new(dout, rows, cols, out_dtype or y.dtype)
    dweights = dout.new_empty((N, K), dtype=_F32)
    rc = (_lib or library()).eb_combine_backward(N, K, cols, dout_ptr, dout_type, lddo, ptr, code, ldy, rows, slots_ptr, weights_ptr, dy_type,
                                                 dy.data_ptr(), lddy, dys_ptr, rows, dweights.data_ptr(), _stream(dout, stream))
    if rc:
        _check(rc)
    return CombineGradient(dy, scales, dweights)


@functools.lru_cache(maxsize=256)
def _gradient_workspace(M, E, N, K):
    return eb_weight_gradient_workspace(M, E, N, K)


@_placed
def weight_gradient(dy, x, offsets=None, tokens=None, dy_scales=None, x_scales=None, out_dtype=None, out=None, accumulate: bool = False,
                    stream=None):
    """Torch convenience for eb_weight_gradient.  ``dy``: device [slots, N], ``x``: [rows, K],
    each of fp16, bf16 or, with its scales, 8 bits; ``offsets``: int32 [E + 1] and
    ``tokens``: int32 [slots], or None, as ``experts.route`` gives them.  Returns [E, N, K],
    without offsets [N, K], of ``out_dtype`` (float32).  ``out``: the output, contiguous or
    with rows further apart; ``accumulate`` adds to it."""
    dy_ptr, dy_type, lddy, dys_ptr, lddys, held = _matrix(dy, "dy", dy_scales)
    x_ptr, x_type, ldx, xs_ptr, ldxs, held_too = _matrix(x, "x", x_scales)
    (M, N), (rows, K), dev = dy.shape, x.shape, dy.get_device()
    if x.get_device() != dev or (out is not None and out.get_device() != dev):
        raise ValueError("x and out must be on dy's GPU")
    if offsets is None:
        E, shape = 1, (N, K)
    else:
        E = offsets.numel() - 1
        if E < 1:
            raise ValueError("offsets must be int32 [E + 1]")
        shape = (E, N, K)
    offsets_ptr, tokens_ptr = _vector(offsets, "offsets", _I32, dev, E + 1), _vector(tokens, "tokens", _I32, dev, M)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out")
        out, ld = dy.new_empty(shape, dtype=out_dtype or _F32), K
    else:
        if out.shape != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError("out must be [E, N, K], without offsets [N, K], of out_dtype")
        ld = ex._pitch(out if offsets is None else out[0], "out")
        if E > 1 and N == 1:
            ld = out.stride(0)
        elif E > 1 and out.stride(0) != N * ld:
            raise ValueError("out's matrices must be stacked row after row")
    out_type = _code(out.dtype)
    if out_type == EB_FP8:
        raise ValueError("the output is fp32, fp16 or bf16")
    nbytes = _gradient_workspace(M, E, N, K)
    work = dy.new_empty((nbytes // 4,), dtype=_F32) if nbytes else None
    rc = (_lib or library()).eb_weight_gradient(
        M, E, N, K, dy_ptr, dy_type, lddy, dys_ptr, lddys, x_ptr, x_type, ldx, rows, xs_ptr, ldxs, tokens_ptr, offsets_ptr, out_type,
        int(accumulate), out.data_ptr(), ld, work.data_ptr() if nbytes else None, nbytes, _stream(dy, stream))
    if rc:
        _check(rc)
    return out


class Saved(NamedTuple):
    """What ``ExpertTraining.forward`` leaves for ``backward``: values in 8 bits with their scales,
    but the experts' rows and what goes by token."""
    route: object      # experts.Route
    scores: object     # fp32 [B, experts]
    x: object          # (values, scales): what the experts read, and the router before it was rounded to 8 bits
    kept: object       # (values, scales) and rstd of the layer norm, or None
    rstd: object
    v: object          # (values, scales) before the activation
    rows: object       # [slots, D] in row_dtype, before they are joined
    read: object = None  # [B, K]: what the router read, under ``exact_router``


class ExpertGradients(NamedTuple):
    """What ``ExpertTraining.backward`` returns; of a layer without norm the last two are None."""
    x: object
    w_up: object        # fp32, as are the others
    w_down: object
    router: object
    norm_weight: object
    norm_bias: object


class ExpertTraining:
    """A mixture of experts in training: ``experts.ExpertLayer``'s two layers behind a layer
    norm, and the gradients of all their weights, from values that wait in 8 bits.

    ``w_up``: [E, N, K], ``w_down``: [E, D, N] (gated [E, D, N / 2]), ``router``: [experts, K]
    fp32 and ``norm_weight``, ``norm_bias``: fp32 [K] (both None: no norm) are the caller's and
    stay so: after a change of ``w_up`` or ``w_down`` call ``refresh``, which makes the 8-bit
    forms that the products take, of each matrix and of its transpose.  ``top``, ``act`` (a
    ReLU or a gated SiLU), ``mode``, ``bias``, ``groups``, ``top_groups``, ``scale``, ``shard_lo``
    and ``row_dtype`` are ``ExpertLayer``'s; of several GPUs' experts a GPU's output, and its
    gradients of x and the router, are shares to be added over the GPUs (and the norm's
    gradients with that of x: where all GPUs hold the same tokens pass the summed dx on).
    The router reads x (behind the norm) unrounded.  Its own gradient is made of x in 8 bits, as the
    experts' are, and of its outputs' gradients in bf16; ``exact_router``: of both as they are, in fp32,
    for which x waits too (a norm's output, else the caller's tensor, to be left as it is until ``backward``).
    Torch records nothing of the calls, also where weights or inputs require gradients, and casts none
    of their products under ``torch.autocast``."""

    def __init__(self, w_up, w_down, router, top: int, act: int = EB_ACT_SILU_GATE, mode: int = ex.EB_SOFTMAX | ex.EB_RENORMALIZE,
                 norm_weight=None, norm_bias=None, eps: float = 1e-5, bias=None, groups: int = 1, top_groups: int = 1, scale: float = 1.0,
                 shard_lo: int = 0, row_dtype=None, exact_router: bool = False):
        if w_up.dim() != 3 or w_down.dim() != 3 or router.dim() != 2:
            raise ValueError("w_up and w_down must be 3-D, router 2-D")
        E, N, K = w_up.shape
        gate = act == EB_ACT_SILU_GATE
        if act not in (EB_ACT_SILU_GATE, ex.EB_ACT_RELU):
            raise ValueError("act must be EB_ACT_RELU or EB_ACT_SILU_GATE")
        if gate and N % 2 or tuple(w_down.shape[::2]) != (E, N // 2 if gate else N) or router.shape[1] != K:
            raise ValueError("w_up [E, N, K], w_down [E, D, N or N / 2] and router [experts, K] do not fit")
        if (norm_weight is None) != (norm_bias is None):
            raise ValueError("norm_weight and norm_bias go together")
        self.w_up, self.w_down, self.router, self.norm_weight, self.norm_bias = w_up, w_down, router, norm_weight, norm_bias
        self.E, self.K, self.D, self.top, self.act, self.mode, self.eps = E, K, int(w_down.shape[1]), top, act, mode, eps
        self.bias, self.groups, self.top_groups, self.scale, self.shard_lo = bias, groups, top_groups, scale, shard_lo
        self.row_dtype, self.exact_router = row_dtype or _BF16, exact_router
        with torch.no_grad(), torch.cuda.device(w_up.device):
            self._up, self._down, self._up_t, self._down_t = (ex.quantize_fp8(w.contiguous(), block_rows=BLOCK) for w in self._forms())

    def _forms(self):
        return self.w_up, self.w_down, self.w_up.transpose(1, 2), self.w_down.transpose(1, 2)

    @torch.no_grad()
    def refresh(self) -> None:
        """The weights' 8-bit forms again, from ``w_up`` and ``w_down`` as they are now: in place,
        so that a captured graph reads the new ones, and may hold the call."""
        with torch.cuda.device(self.w_up.device):
            for w, (q, scales) in zip(self._forms(), (self._up, self._down, self._up_t, self._down_t)):
                if w.shape != q.shape or w.device != q.device:
                    raise ValueError("w_up and w_down must keep their shapes and GPU")
                w = w.contiguous()
                E, rows, cols = w.shape
                ex.eb_quantize_fp8(E, rows, cols, w.data_ptr(), _code(w.dtype), cols, BLOCK, q.data_ptr(), cols + 15 & -16,
                                   scales.data_ptr(), 0, _stream(w, None))

    @torch.no_grad()
    def forward(self, x, out_dtype=None):
        """``x``: device [B, K] of fp32, fp16 or bf16.  Returns (out [B, D] of ``out_dtype``
        (float32), Saved)."""
        if x.dim() != 2 or x.shape[1] != self.K or not x.is_cuda:
            raise ValueError("x must be [B, K] on the GPU")
        with torch.cuda.device(x.device), torch.autocast("cuda", enabled=False):
            kept = rstd = None
            if self.norm_weight is not None:
                n = layer_norm(x, self.norm_weight, self.norm_bias, self.eps, out_dtype=x.dtype, checkpoint=True)
                x, kept, rstd = n.y, (n.kept, n.kept_scales), n.rstd
            scores = x.float() @ self.router.t()
            r = ex.route(scores, self.top, self.mode, self.bias, self.groups, self.top_groups, self.scale, self.shard_lo, self.shard_lo + self.E)
            q = ex.quantize_fp8(x)
            v = ex.product(*q, *self._up, r.offsets, r.tokens, out_dtype=_FP8)
            h = activation(*v, act=self.act, out_dtype=_FP8)
            rows = ex.product(*h, *self._down, r.offsets, out_dtype=self.row_dtype)
            out = combine(rows, r.slots, r.weights, out_dtype=out_dtype or _F32)
        return out, Saved(r, scores, q, kept, rstd, v, rows, x if self.exact_router else None)

    def backward(self, saved: Saved, dout, dx_dtype=None) -> ExpertGradients:
        """``dout``: [B, D] of fp32, fp16 or bf16, the gradient of forward's output; ``dx_dtype``: the
        type of x's gradient, and of the rows from which the norm's are made (behind a norm bf16,
        else fp32)."""
        return self._backward(saved, dout, dx_dtype)[0]

    @torch.no_grad()
    def _backward(self, saved, dout, dx_dtype=None):
        r = saved.route
        dx_dtype = dx_dtype or (_F32 if self.norm_weight is None else _BF16)
        if _code(dx_dtype) == EB_FP8:
            raise ValueError("dx_dtype must be fp32, fp16 or bf16")
        with torch.cuda.device(dout.device), torch.autocast("cuda", enabled=False):
            g = combine_backward(dout, saved.rows, r.slots, r.weights, out_dtype=_FP8)
            dz = (g.dy, g.dy_scales)
            dh = ex.product(*dz, *self._down_t, r.offsets, out_dtype=_BF16)
            dv = activation_backward(dh, *saved.v, act=self.act, out_dtype=_FP8)
            h = activation(*saved.v, act=self.act, out_dtype=_FP8)  # forward's, made again
            w_down = weight_gradient(dz[0], h[0], r.offsets, dy_scales=dz[1], x_scales=h[1])
            w_up = weight_gradient(dv[0], saved.x[0], r.offsets, r.tokens, dy_scales=dv[1], x_scales=saved.x[1])
            dslots = ex.product(*dv, *self._up_t, r.offsets, out_dtype=_BF16)
            # In bf16, whose range is fp32's: the rows' gradients before they are joined (each comes of
            # 4-bit values) and, unless more is asked for, what the router's gradient and the norm's take.
            dscores = self._dscores(saved, g.dweights)
            dx = combine(dslots, r.slots, out_dtype=_F32) + dscores @ self.router
            if saved.read is not None:
                router = dscores.t() @ saved.read.float()
            else:
                router = weight_gradient(dscores.to(_BF16), saved.x[0], x_scales=saved.x[1])
            dx = dx.to(dx_dtype)
            norm_weight = norm_bias = None
            if self.norm_weight is not None:
                dx, norm_weight, norm_bias = layer_norm_backward(dx, saved.kept[0], saved.rstd, x_scales=saved.kept[1],
                                                                 weight=self.norm_weight)
        return ExpertGradients(dx, w_up, w_down, router, norm_weight, norm_bias), dict(dz=dz, dh=dh, dv=dv, h=h, dslots=dslots, dweights=g.dweights, dscores=dscores)

    def _dscores(self, saved, dweights):
        """The router's outputs' gradient from that of the chosen pairs' weights (0 for other GPUs' pairs).

        With EB_RENORMALIZE a token's weights w are its own chosen experts' alone, whose scores may lie
        far below others' that a bias or a group keeps out: no sum over those is divided by.
        softmax: w (d - sum of w d); sigmoid: that times 1 - p.  Scores are what the route takes them
        as: an infinity the largest float, NaN minus infinity."""
        scores, ids = saved.scores.nan_to_num(-math.inf, torch.finfo(_F32).max, -math.inf), saved.route.ids
        at, there = ids.clamp(min=0).long(), ids >= 0
        sigmoid = self.mode & 0xFF == ex.EB_SIGMOID
        d = torch.where(there, dweights * self.scale, 0.0)
        x = scores.gather(1, at)
        if self.mode & ex.EB_RENORMALIZE:
            most = torch.where(there, x, torch.finfo(_F32).min).amax(1, keepdim=True)
            if sigmoid:  # e^-m / (1 + e^-x): no underflow where all x are low
                m = most.clamp(max=0)
                w = torch.where(there, 1 / (torch.exp(m) + torch.exp(m - x)), 0.0)
            else:
                w = torch.where(there, torch.exp(x - most), 0.0)
            w = w / torch.where(there.any(1, keepdim=True), w.sum(1, keepdim=True), 1.0)
            d = w * (d - (w * d).sum(1, keepdim=True))
            if sigmoid:
                d = d * torch.sigmoid(-x)
        elif sigmoid:
            d = d * torch.sigmoid(x) * torch.sigmoid(-x)
        ds = torch.zeros_like(scores).scatter_add_(1, at, d)
        if sigmoid or self.mode & ex.EB_RENORMALIZE:
            return ds
        p = torch.softmax(scores, 1).nan_to_num(0.0)  # without an expert to choose none has a share
        return p * (ds - (ds * p).sum(1, keepdim=True))
