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
from typing import NamedTuple

from . import eb, experts as ex
from .eb import EB_BF16, EB_F16, EB_F32, _check
from .experts import BLOCK, EB_ACT_RELU, EB_ACT_SILU_GATE, EB_FP8, _code, _gpu, _place, _raw_stream, _same_device

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


def _placed(f):
    """The call under its ``stream``, or on its first tensor's GPU: at once where that is current."""
    @functools.wraps(f)
    def call(x, *args, stream=None, **kw):
        if stream is None and -1 < x.get_device() == _gpu():
            return f(x, *args, **kw)
        if not x.is_cuda:
            raise ValueError("expected device tensors")
        import torch

        with _place(torch, x, stream):
            return f(x, *args, stream=stream, **kw)
    return call


def _stream(x, stream):
    return _raw_stream(x.get_device()) if stream is None else stream.cuda_stream


def _matrix(x, what: str, scales=None, cols: int | None = None):
    """(pointer, code, pitch, scales' pointer, scales' pitch, what has to live on) of a 2-D
    tensor with unit column stride, in 8 bits with its scales."""
    if x.dim() != 2:
        raise ValueError(f"{what} must be 2-D")
    code = _code(x.dtype, fp8=True)
    rows, n = x.shape
    if cols is not None and n != cols:
        raise ValueError(f"{what} must have {cols} columns")
    ld = ex._pitch(x, what)
    if code != EB_FP8:
        if scales is not None:
            raise ValueError(f"{what} is not in 8 bits: it takes no scales")
        return x.data_ptr(), code, ld, None, 0, x
    if rows == 1 and ld % 16:
        ld = ld + 15 & -16  # a single row has no next one
    blocks = (n + BLOCK - 1) // BLOCK
    if scales is None or str(scales.dtype) != "torch.float32" or scales.shape != (rows, blocks):
        raise ValueError(f"{what} in 8 bits needs its scales, fp32 [rows, ceil(columns/128)]")
    by_row, by_block = scales.stride()
    if rows > 1 and by_row != 1 or blocks > 1 and by_block < rows:
        scales = scales.t().contiguous().t()
        by_block = rows
    return x.data_ptr(), code, ld, scales.data_ptr(), by_block if blocks > 1 else rows, scales


def _new(like, rows: int, cols: int, dtype):
    """An output matrix of rows x cols beside ``like``: (tensor, code, pitch, scales or None)."""
    import torch

    code = _code(dtype, fp8=True)
    if code != EB_FP8:
        return like.new_empty((rows, cols), dtype=dtype), code, cols, None
    ld = cols + 15 & -16
    q = like.new_empty((rows, ld), dtype=dtype)
    scales = like.new_empty_strided((rows, (cols + BLOCK - 1) // BLOCK), (1, rows), dtype=torch.float32)
    return (q if ld == cols else q[:, :cols]), code, ld, scales


def _floats(x, what: str, dev, *shape):
    """The address of a contiguous fp32 tensor of a shape on a GPU; None of None."""
    if x is None:
        return None
    if str(x.dtype) != "torch.float32" or x.shape != shape or not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous fp32 {list(shape)}")
    _same_device(dev, x)
    return x.data_ptr()


def _ints(x, what: str, dev, *shape):
    """The same for int32."""
    if x is None:
        return None
    if str(x.dtype) != "torch.int32" or x.shape != shape or not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous int32 {list(shape)}")
    _same_device(dev, x)
    return x.data_ptr()


def _bf16():
    import torch

    return torch.bfloat16


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
    import torch

    ptr, code, ldx, *_ = _matrix(x, "x")
    if code == EB_FP8:
        raise ValueError("x must be fp32, fp16 or bf16")
    (rows, cols), dev = x.shape, x.device
    y, out_type, ldy, y_scales = _new(x, rows, cols, out_dtype or torch.bfloat16)
    mean = rstd = kept = kept_scales = None
    ldk = 0
    if statistics:
        mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind(0)
    elif checkpoint:
        rstd = x.new_empty((rows,), dtype=torch.float32)
    if checkpoint:
        kept, _, ldk, kept_scales = _new(x, rows, cols, torch.float8_e4m3fn)
    rc = (_lib or library()).eb_layer_norm(
        rows, cols, ptr, code, ldx, _floats(weight, "weight", dev, cols), _floats(bias, "bias", dev, cols), eps, out_type, y.data_ptr(), ldy,
        None if y_scales is None else y_scales.data_ptr(), rows, None if kept is None else kept.data_ptr(), ldk,
        None if kept is None else kept_scales.data_ptr(), rows, None if mean is None else mean.data_ptr(),
        None if rstd is None else rstd.data_ptr(), _stream(x, stream))
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
    import torch

    dy_ptr, dy_type, lddy, *_ = _matrix(dy, "dy")
    if dy_type == EB_FP8:
        raise ValueError("dy must be fp32, fp16 or bf16")
    (rows, cols), dev = dy.shape, dy.device
    if x.shape != dy.shape:
        raise ValueError("x must have dy's shape")
    x_ptr, x_type, ldx, xs_ptr, ldxs, held = _matrix(x, "x", x_scales)
    _same_device(dev, x, x_scales)
    if (x_type == EB_FP8) != (mean is None):
        raise ValueError("mean goes with an x in floating point, and only with that")
    dx = dy.new_empty((rows, cols))
    dweight = dbias = work = None
    nbytes = 0
    if parameters:
        dweight, dbias = dy.new_empty((2, cols), dtype=torch.float32).unbind(0)
        nbytes = _norm_workspace(rows, cols)
        work = dy.new_empty((nbytes // 4,), dtype=torch.float32)
    rc = (_lib or library()).eb_layer_norm_backward(
        rows, cols, dy_ptr, dy_type, lddy, x_ptr, x_type, ldx, xs_ptr, ldxs, _floats(mean, "mean", dev, rows), _floats(rstd, "rstd", dev, rows),
        _floats(weight, "weight", dev, cols), dx.data_ptr(), cols, None if work is None else dweight.data_ptr(),
        None if work is None else dbias.data_ptr(), None if work is None else work.data_ptr(), nbytes, _stream(dy, stream))
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
    _same_device(v.device, v_scales)
    rows = v.shape[0]
    h, out_type, ldh, scales = _new(v, rows, cols, out_dtype or _bf16())
    rc = (_lib or library()).eb_activation(rows, cols, act, ptr, code, ldv, vs_ptr, ldvs, out_type, h.data_ptr(), ldh,
                                           None if scales is None else scales.data_ptr(), rows, _stream(v, stream))
    if rc:
        _check(rc)
    return h if scales is None else (h, scales)


@_placed
def activation_backward(dh, v, v_scales=None, act: int = EB_ACT_SILU_GATE, out_dtype=None, stream=None):
    """Torch convenience for eb_activation_backward.  ``dh``: device [rows, cols] of fp32,
    fp16 or bf16; ``v``, ``v_scales``, ``act``: forward's.  Returns dv, of v's shape and of
    ``out_dtype`` (bfloat16), or for float8_e4m3fn (dv, scales)."""
    cols = _width_of_v(v, act)
    dh_ptr, dh_type, lddh, *_ = _matrix(dh, "dh", cols=cols)
    if dh_type == EB_FP8:
        raise ValueError("dh must be fp32, fp16 or bf16")
    rows = dh.shape[0]
    if v.shape[0] != rows:
        raise ValueError("v must have dh's rows")
    ptr, code, ldv, vs_ptr, ldvs, held = _matrix(v, "v", v_scales)
    _same_device(dh.device, v, v_scales)
    dv, out_type, lddv, scales = _new(dh, rows, v.shape[1], out_dtype or _bf16())
    rc = (_lib or library()).eb_activation_backward(rows, cols, act, dh_ptr, dh_type, lddh, ptr, code, ldv, vs_ptr, ldvs, out_type,
                                                    dv.data_ptr(), lddv, None if scales is None else scales.data_ptr(), rows,
                                                    _stream(dh, stream))
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
    (rows, cols), M = x.shape, tokens.numel()
    tokens_ptr = _ints(tokens, "tokens", x.device, M)
    _same_device(x.device, x_scales, out)
    scales = None
    if out is None:
        out, _, ldo, scales = _new(x, M, cols, x.dtype)
    else:
        if code == EB_FP8:
            raise ValueError("out is for floating-point rows")
        if out.dtype != x.dtype or out.shape != (M, cols):
            raise ValueError("out must be [slots, cols] of x's type")
        ldo = ex._pitch(out, "out")
    rc = (_lib or library()).eb_dispatch(M, cols, ptr, code, ldx, rows, xs_ptr, ldxs, tokens_ptr, out.data_ptr(), ldo,
                                         None if scales is None else scales.data_ptr(), M, _stream(x, stream))
    if rc:
        _check(rc)
    return out if scales is None else (out, scales)


@_placed
def combine(y, slots, weights=None, out_dtype=None, stream=None):
    """Torch convenience for eb_combine.  ``y``: device [rows, cols] of fp32, fp16 or bf16;
    ``slots``: int32 [tokens, K] as ``experts.route`` gives them; ``weights``: fp32
    [tokens, K] or None.  Returns [tokens, cols] of ``out_dtype`` (y's type)."""
    ptr, code, ldy, *_ = _matrix(y, "y")
    if code == EB_FP8 or slots.dim() != 2:
        raise ValueError("y must be fp32, fp16 or bf16, slots 2-D")
    (rows, cols), (N, K), dev = y.shape, slots.shape, y.device
    slots_ptr, weights_ptr = _ints(slots, "slots", dev, N, K), _floats(weights, "weights", dev, N, K)
    out = y.new_empty((N, cols), dtype=out_dtype or y.dtype)
    rc = (_lib or library()).eb_combine(N, K, cols, ptr, code, ldy, rows, slots_ptr, weights_ptr, _code(out.dtype), out.data_ptr(), cols,
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
    import torch

    dout_ptr, dout_type, lddo, *_ = _matrix(dout, "dout")
    ptr, code, ldy, *_ = _matrix(y, "y", cols=dout.shape[1])
    if EB_FP8 in (code, dout_type) or slots.dim() != 2 or slots.shape[0] != dout.shape[0]:
        raise ValueError("dout and y must be fp32, fp16 or bf16, slots [tokens, K]")
    (N, K), (rows, cols), dev = slots.shape, y.shape, dout.device
    _same_device(dev, y)
    slots_ptr, weights_ptr = _ints(slots, "slots", dev, N, K), _floats(weights, "weights", dev, N, K)
    dy, dy_type, lddy, scales = _new(dout, rows, cols, out_dtype or y.dtype)
    dweights = dout.new_empty((N, K), dtype=torch.float32)
    rc = (_lib or library()).eb_combine_backward(N, K, cols, dout_ptr, dout_type, lddo, ptr, code, ldy, rows, slots_ptr, weights_ptr, dy_type,
                                                 dy.data_ptr(), lddy, None if scales is None else scales.data_ptr(), rows,
                                                 dweights.data_ptr(), _stream(dout, stream))
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
    import torch

    if dy.dim() != 2 or x.dim() != 2:
        raise ValueError("dy and x must be 2-D")
    (M, N), (rows, K), dev = dy.shape, x.shape, dy.device
    dy_ptr, dy_type, lddy, dys_ptr, lddys, held = _matrix(dy, "dy", dy_scales)
    x_ptr, x_type, ldx, xs_ptr, ldxs, held_too = _matrix(x, "x", x_scales)
    _same_device(dev, x, dy_scales, x_scales, out)
    if offsets is not None and (offsets.dim() != 1 or offsets.numel() < 2):
        raise ValueError("offsets must be int32 [E + 1]")
    E = 1 if offsets is None else offsets.numel() - 1
    offsets_ptr, tokens_ptr = _ints(offsets, "offsets", dev, E + 1), _ints(tokens, "tokens", dev, M)
    shape = (N, K) if offsets is None else (E, N, K)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out")
        out, ld = dy.new_empty(shape, dtype=out_dtype or torch.float32), K
    else:
        if out.shape != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError("out must be [E, N, K], without offsets [N, K], of out_dtype")
        ld = ex._pitch(out if offsets is None else out[0], "out")
        if E > 1 and N == 1:
            ld = out.stride(0)
        elif E > 1 and out.stride(0) != N * ld:
            raise ValueError("out's matrices must be stacked row after row")
    nbytes = _gradient_workspace(M, E, N, K)
    work = dy.new_empty((nbytes // 4,), dtype=torch.float32) if nbytes else None
    rc = (_lib or library()).eb_weight_gradient(
        M, E, N, K, dy_ptr, dy_type, lddy, dys_ptr, lddys, x_ptr, x_type, ldx, rows, xs_ptr, ldxs, tokens_ptr, offsets_ptr, _code(out.dtype),
        int(accumulate), out.data_ptr(), ld, work.data_ptr() if nbytes else None, nbytes, _stream(dy, stream))
    if rc:
        _check(rc)
    return out
