"""The root-mean-square norm that stands behind an all-reduce, with the residual's addition, into 16 bits or 8-bit codes with scales.  The
front end of fc_rms_norm and fc_rms_norm_quantize (include/fc.h has the formulas).

x, residual and the results are float16 or bfloat16 tensors [tokens, hidden] whose last axis is dense, rows at any stride that is a
multiple of 8 elements.  Every call is asynchronous on ``torch.cuda.current_stream()``, allocates nothing with its results given and can be
captured into a HIP graph.  Serving only: tensors that require a gradient are refused unless gradients are off.
"""
from __future__ import annotations

from . import binding
from .attention import _type
from .binding import QUANTIZER_SYM, _check, _coded_outputs, _dev, _meet, _shape, _stream, _torch

_F32 = 2                                                 # FC_TYPE_F32


def _no_gradient(t, what):
    if t.requires_grad and _torch().is_grad_enabled():
        raise ValueError("%s requires a gradient, which no norm records: call it under torch.no_grad(), or on %s.detach()" % (what, what))


def _row(t, what, dtype=None, shape=None):
    """a [tokens, hidden] activation on the current device, in 128-bit units"""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor; this library has no CPU path" % what)
    if dtype is None:
        _type(t, what)
    elif t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if t.dim() != 2:
        raise ValueError("%s must be [tokens, hidden], got shape %s" % (what, tuple(t.shape)))
    if shape is not None:
        _shape(t, shape, what)
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s lives on %s but the current device is cuda:%d; the C ABI works on the current device"
                         % (what, t.device, torch.cuda.current_device()))
    _no_gradient(t, what)
    if t.numel() and (t.stride(1) != 1 or (t.shape[0] > 1 and t.stride(0) % 8) or t.data_ptr() % 16):
        raise ValueError("%s must have a dense last axis, a row stride that is a multiple of 8 elements and a 16-byte aligned start, "
                         "got strides %s" % (what, tuple(t.stride())))
    return t


def _stride(t):
    return t.stride(0) if t.shape[0] > 1 else 0


def _result(out, x, what):
    if out is None:
        return _torch().empty(tuple(x.shape), dtype=x.dtype, device=x.device)
    _row(out, what, x.dtype, tuple(x.shape))
    if out.shape[0] > 1 and out.stride(0) < out.shape[1]:
        raise ValueError("%s must not overlap itself, got strides %s" % (what, tuple(out.stride())))
    return out


def _inputs(x, weight, residual, sum_out):
    """(weight's type, address and stride of the residual, the sum or None) of checked tensors"""
    torch = _torch()
    _row(x, "x")
    if isinstance(weight, torch.Tensor) and weight.dtype not in (x.dtype, torch.float32):
        raise TypeError("weight must be of x's type or float32, got %s" % weight.dtype)
    _dev(weight, getattr(weight, "dtype", None), "weight")
    _shape(weight, (x.shape[1],), "weight")
    _no_gradient(weight, "weight")
    if weight.data_ptr() % 16:
        raise ValueError("weight must begin on a 16-byte boundary")
    kind = _F32 if weight.dtype == torch.float32 else _type(weight, "weight")
    if residual is None:
        if sum_out is not None:
            raise ValueError("sum_out goes with a residual")
        return kind, (None, 0), None
    _row(residual, "residual", x.dtype, tuple(x.shape))
    return kind, (residual.data_ptr(), _stride(residual)), _result(sum_out, x, "sum_out")


def _apart(results, x, residual, weight):
    """results, (what, tensor, whether it may be x or residual), overlap neither each other nor what is read: workgroups take the rows in any order"""
    for i, (what, t, in_place) in enumerate(results):
        for other, u in (("x", x), ("residual", residual), ("weight", weight)):
            if u is None or not _meet(t, u):
                continue
            if not (in_place and other != "weight" and t.data_ptr() == u.data_ptr() and _stride(t) == _stride(u)):
                raise ValueError("%s must not overlap %s%s" % (what, other, ", unless it has the same rows" if in_place and other != "weight" else ""))
        for other, u, _ in results[:i]:
            if _meet(t, u):
                raise ValueError("%s and %s need memory of their own" % (other, what))


def rms_norm(x, weight, eps: float = 1e-5, residual=None, out=None, sum_out=None):
    """fc_rms_norm: y, the norm of x's rows times weight (of x's type or float32, [hidden]).  With a residual: (y, sum), the norm of
    x + residual and that sum, which the next layer's residual is.  out and sum_out may be x or residual, row for row; what overlaps
    otherwise is refused."""
    done = (binding._native or binding._calls()).rms_norm(x, weight, eps, residual, out, sum_out)
    if done is not None:
        return done
    kind, other, total = _inputs(x, weight, residual, sum_out)
    y = _result(out, x, "out")
    _apart([(what, t, True) for what, t in (("out", out), ("sum_out", sum_out)) if t is not None], x, residual, weight)
    _check(binding.lib().fc_rms_norm(x.data_ptr(), _stride(x), *other, weight.data_ptr(), kind, x.shape[0], x.shape[1], eps, _type(x, "x"),
                                     *((None, 0) if total is None else (total.data_ptr(), _stride(total))), y.data_ptr(), _stride(y), _stream()),
           "fc_rms_norm")
    return y if total is None else (y, total)


def rms_norm_quantize(x, weight, eps: float = 1e-5, group: int = 128, quantizer: int = QUANTIZER_SYM, residual=None, out=None, sum_out=None):
    """fc_rms_norm_quantize: (codes uint8 [tokens, hidden], scales float32 [tokens, hidden / group]) of the norm, as quantize_sym (8 bit) and
    quantize_fp8 have them, and with a residual the sum x + residual behind them.  group: a power of two in [32, 16384], or hidden: one
    scale a token.  dequantize_sym and dequantize_fp8 read codes in groups of a power of two."""
    done = (binding._native or binding._calls()).rms_norm_quantize(x, weight, eps, group, quantizer, residual, out, sum_out)
    if done is not None:
        return done
    torch = _torch()
    kind, other, total = _inputs(x, weight, residual, sum_out)
    tokens, hidden = x.shape
    if group < 1 or hidden % group or (group != hidden and (group < 32 or group > 16384 or group & (group - 1))):
        raise binding.FcError(-3, "fc_rms_norm_quantize")
    codes, scales = _coded_outputs(x.device, tokens, hidden, group, 8, out, [(torch.float32, "scales")])
    _apart([("codes (out)", codes, False), ("scales (out)", scales, False)] * (out is not None) + [("sum_out", total, True)] * (sum_out is not None), x, residual,
           weight)
    _check(binding.lib().fc_rms_norm_quantize(x.data_ptr(), _stride(x), *other, weight.data_ptr(), kind, tokens, hidden, eps, _type(x, "x"), group,
                                              quantizer, *((None, 0) if total is None else (total.data_ptr(), _stride(total))), codes.data_ptr(),
                                              scales.data_ptr(), _stream()), "fc_rms_norm_quantize")
    return (codes, scales) if total is None else (codes, scales, total)
