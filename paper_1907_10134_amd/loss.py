"""ctypes binding of the loss against a teacher's top logits (bppsa_distil in include/bppsa.h)."""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple

import torch

from .binding import _aside, _check, _lib
from .ssm import _TYPES, _f32, _here, _i32, _like, _pack_rows, _param, _rows, _whole

_c_int, _c_void_p = ctypes.c_int, ctypes.c_void_p
_lib.bppsa_distil.restype = _c_int
_lib.bppsa_distil.argtypes = [_c_void_p] * 4

_pack_distil = struct.Struct("@6iPqq" + "P" * 5 + "2f").pack

DistilLoss = namedtuple("DistilLoss", "loss dlogits")


def distil(logits, top_logits, top_index, temperature=1.0, top_norm=None, targets=None, hard=0.0, weight=None, gradient=True,
           loss=None, dlogits=None, stream=None):
    """bppsa_distil: the loss [T, B] of each row and, with `gradient`, the gradient of their sum for the logits, as DistilLoss.

    logits [T, B, V] float32, bfloat16 or float16, the V logits side by side; top_logits [T, B, K] of any of these types and
    top_index [T, B, K] int32: the teacher's entries, those with an index of -1 left out; top_norm [T, B] float32, the
    teacher's logsumexp of its logits / temperature: makes all other tokens one more class; targets [T, B] int32 (-1: none) with
    the share `hard` of the loss; weight [T, B] float32: of each row, those of weight 0 are not read.  dlogits may be `logits`
    itself, whose place the gradient then takes.  All of them may also be without the dimension of the samples, [rows, ...]."""
    if stream is not None:
        return _aside(stream, distil, logits, top_logits, top_index, temperature, top_norm, targets, hard, weight, gradient, loss,
                      dlogits)
    if not (isinstance(logits, torch.Tensor) and isinstance(top_logits, torch.Tensor) and isinstance(top_index, torch.Tensor)):
        raise TypeError("logits, top_logits and top_index must be torch.Tensors")
    t, shape, at = logits.dtype, logits.shape, logits.get_device()
    if len(shape) not in (2, 3):
        raise ValueError("logits must be [T, B, V] or [rows, V]")
    if t not in _TYPES or top_logits.dtype not in _TYPES:
        raise ValueError("logits and top_logits must be float32, bfloat16 or float16")
    if top_logits.dim() != len(shape) or top_logits.shape[:-1] != shape[:-1]:
        raise ValueError("top_logits must have shape %s and K, got %s" % (tuple(shape[:-1]), tuple(top_logits.shape)))
    rows, entries = shape[:-1], top_logits.shape
    V, K = shape[-1], entries[-1]
    wide = (lambda x, name: _rows(x, shape, t, name, at)) if len(shape) == 3 else \
        (lambda x, name: _rows(x.unsqueeze(1) if isinstance(x, torch.Tensor) else x, (shape[0], 1, V), t, name, at))
    if hard and targets is None:
        raise ValueError("distil: hard = %r needs targets" % (hard,))
    T, B = (rows[0], rows[1]) if len(shape) == 3 else (rows[0], 1)
    if not top_logits.is_contiguous():
        raise ValueError("top_logits must be contiguous")
    packed = _pack_distil(T, B, V, K, _TYPES[t], _TYPES[top_logits.dtype], *wide(logits, "logits"),
                          _whole(top_logits, top_logits.dtype, "top_logits", at), _param(top_index, entries, "top_index", at, _i32),
                          _param(top_norm, rows, "top_norm", at), _param(weight, rows, "weight", at),
                          _param(targets, rows, "targets", at, _i32), float(temperature), float(hard))
    if loss is None:
        loss = torch.empty(rows, dtype=_f32, device=logits.device)
    elif not isinstance(loss, torch.Tensor):
        raise TypeError("loss must be a torch.Tensor")
    out = None
    if dlogits is not None or gradient:
        if dlogits is None:
            dlogits = _like(logits)
        out = _pack_rows(*wide(dlogits, "dlogits"))
    _check(_lib.bppsa_distil(packed, _param(loss, rows, "loss", at), out, _here(at)), "bppsa_distil")
    return DistilLoss(loss, dlogits)
