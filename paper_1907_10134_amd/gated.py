"""ctypes binding of the gated linear recurrence: over sequences, its gradients and its step for single tokens, with the names of
the C ABI in include/bppsa.h.

Activations are float32, bfloat16 or float16, all of one call the same, [T, B, D] with the channels contiguous and any strides
of time and sample; parameters, states and their gradients are contiguous float32.  A call runs on the current stream or on
`stream`; the caller orders that stream with the ones that make the inputs and use the results.
"""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple

import torch

from .binding import _aside, _check, _lib
from .ssm import (_NONE, _TYPES, _f32, _here, _i32, _like, _opaque, _output, _own, _pack_rows, _param, _rows, _slots,
                  _token_output, _whole)

_c_int, _c_void_p, _c_size_t = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
for _name, _res, _args in (
        ("bppsa_gated_scan_states_bytes", _c_size_t, [_c_int] * 3),
        ("bppsa_gated_scan_workspace_bytes", _c_size_t, [_c_int] * 3),
        ("bppsa_gated_scan", _c_int, [_c_void_p] * 5 + [_c_size_t, _c_void_p]),
        ("bppsa_gated_scan_backward_workspace_bytes", _c_size_t, [_c_int] * 3),
        ("bppsa_gated_scan_backward", _c_int, [_c_void_p] * 6 + [_c_size_t, _c_void_p]),
        ("bppsa_gated_scan_step", _c_int, [_c_void_p] * 3 + [_c_int] + [_c_void_p] * 2)):
    getattr(_lib, _name).restype = _res
    getattr(_lib, _name).argtypes = _args

_pack_layer = struct.Struct("@4i" + "Pqq" * 4 + "P" * 5).pack
_pack_grads = struct.Struct("@" + "Pqq" * 4 + "P" * 4).pack


def _quick_layer(token, x, r, i, decay, z, r_bias, i_bias, h0, lengths):
    """_layer in one go where every tensor is as it should be with nothing odd about it; None otherwise."""
    try:
        t, shape, at = x.dtype, x.shape, x.get_device()
        if token:
            (B, D), T = shape, 1
        else:
            T, B, D = shape
        if not (r.dtype is t and i.dtype is t and decay.dtype is _f32 and r.shape == shape and i.shape == shape and
                decay.shape == (D,) and at >= 0 and r.get_device() == at and i.get_device() == at and
                decay.get_device() == at and decay.is_contiguous()):
            return None
        sx, sr, si = x.stride(), r.stride(), i.stride()
        if not sx[-1] == sr[-1] == si[-1] == 1:
            return None
        pz, sz = 0, sx
        if z is not None:
            sz = z.stride()
            if not (z.dtype is t and z.get_device() == at and z.shape == shape and sz[-1] == 1):
                return None
            pz = z.data_ptr()
        params = (decay.data_ptr(), _own(r_bias, (D,), at), _own(i_bias, (D,), at), _own(h0, (B, D), at))
        if None in params:
            return None
        ends = 0 if lengths is None else _param(lengths, (B,), "lengths", at, _i32)
        kind = _TYPES[t]
        if token:
            return _pack_layer(1, B, D, kind, x.data_ptr(), 0, sx[0], r.data_ptr(), 0, sr[0], i.data_ptr(), 0, si[0], pz, 0, sz[0],
                               *params, ends), (1, B, D), at
        return _pack_layer(T, B, D, kind, x.data_ptr(), sx[0], sx[1], r.data_ptr(), sr[0], sr[1], i.data_ptr(), si[0], si[1], pz,
                           sz[0], sz[1], *params, ends), (T, B, D), at
    except (AttributeError, KeyError, TypeError, ValueError):
        return None


def _layer(token, x, r, i, decay, z, r_bias, i_bias, h0=None, lengths=None):
    """The bytes of bppsa_gated, (T, B, D) and the device's number; token: of [B, D], T = 1."""
    quick = _quick_layer(token, x, r, i, decay, z, r_bias, i_bias, h0, lengths)
    if quick is not None:
        return quick
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a torch.Tensor")
    if token:
        if x.dim() != 2:
            raise ValueError("x must be [B, D]")
        one = lambda t: t.unsqueeze(0) if isinstance(t, torch.Tensor) else t
        return _layer(False, one(x), one(r), one(i), decay, one(z), r_bias, i_bias)
    if x.dim() != 3:
        raise ValueError("x must be [T, B, D]")
    (T, B, D), t, shape, at = x.shape, x.dtype, x.shape, x.get_device()
    if t not in _TYPES:
        raise ValueError("activations must be float32, bfloat16 or float16, got %s" % t)
    if decay is None:
        raise TypeError("decay must be a torch.Tensor")
    return _pack_layer(T, B, D, _TYPES[t], *_rows(x, shape, t, "x", at), *_rows(r, shape, t, "r", at), *_rows(i, shape, t, "i", at),
                       *(_NONE if z is None else _rows(z, shape, t, "z", at)), _param(decay, (D,), "decay", at),
                       _param(r_bias, (D,), "r_bias", at), _param(i_bias, (D,), "i_bias", at), _param(h0, (B, D), "h0", at),
                       _param(lengths, (B,), "lengths", at, _i32)), (T, B, D), at


def gated_scan_workspace_bytes(T, B, D):
    return int(_lib.bppsa_gated_scan_workspace_bytes(T, B, D))


def gated_scan_states(T, B, D, device="cuda"):
    """The array that gated_scan(states=) fills for gated_scan_backward: bppsa_gated_scan_states_bytes(T, B, D) bytes."""
    n = int(_lib.bppsa_gated_scan_states_bytes(T, B, D))
    if not n:
        raise ValueError("gated_scan_states: no such sizes (%d, %d, %d)" % (T, B, D))
    return torch.empty(n, dtype=torch.uint8, device=device)


def _states(states, dims, device):
    if states is None:
        return None
    at = _whole(states, torch.uint8, "states", device)
    if states.numel() < _lib.bppsa_gated_scan_states_bytes(*dims):
        raise ValueError("states is too small for these sizes")
    return at


def gated_scan(x, r, i, decay, z=None, r_bias=None, i_bias=None, h0=None, lengths=None, y=None, h_last=None, states=None,
               workspace=None, stream=None):
    """bppsa_gated_scan: y [T, B, D] of the recurrence whose decay is exp(-decay sigmoid(r + r_bias)), into which
    sigmoid(i + i_bias) x enters.

    x, r, i, z [T, B, D]; decay, r_bias, i_bias [D]; h0 [B, D]; lengths [B] int32.  h_last [B, D] receives the last states,
    states (see gated_scan_states) what gated_scan_backward needs."""
    if stream is not None:
        return _aside(stream, gated_scan, x, r, i, decay, z, r_bias, i_bias, h0, lengths, y, h_last, states, workspace)
    layer, dims, at = _layer(False, x, r, i, decay, z, r_bias, i_bias, h0, lengths)
    y, out = _output(y, x, "y", at)
    _ws, ws, nbytes = _opaque(workspace, _lib.bppsa_gated_scan_workspace_bytes(*dims), at)
    _check(_lib.bppsa_gated_scan(layer, out, _param(h_last, dims[1:], "h_last", at), _states(states, dims, at), ws, nbytes,
                                 _here(at)), "bppsa_gated_scan")
    return y


GatedGrads = namedtuple("GatedGrads", "dx dr di ddecay dz dr_bias di_bias dh0")


def gated_scan_backward_workspace_bytes(T, B, D):
    return int(_lib.bppsa_gated_scan_backward_workspace_bytes(T, B, D))


def gated_scan_backward(dy, x, r, i, decay, states, z=None, r_bias=None, i_bias=None, h0=None, lengths=None, dh_last=None,
                        dh0=None, workspace=None, stream=None):
    """bppsa_gated_scan_backward: the gradients of sum(y dy) + sum(h_last dh_last), as GatedGrads; the other arguments are those
    of the gated_scan call that filled `states`.  dz, dr_bias and di_bias are None where there is no such input; dh0 [B, D] is
    filled if given."""
    if stream is not None:
        return _aside(stream, gated_scan_backward, dy, x, r, i, decay, states, z, r_bias, i_bias, h0, lengths, dh_last, dh0,
                      workspace)
    layer, dims, at = _layer(False, x, r, i, decay, z, r_bias, i_bias, h0, lengths)
    if states is None:
        raise TypeError("states must be the array that gated_scan filled")
    made = [None if t is None else _like(t) for t in (x, r, i, z)]
    like = lambda t: None if t is None else torch.empty_like(t)
    ddecay, drb, dib = like(decay), like(r_bias), like(i_bias)
    rows = []
    for t in made:
        rows += _NONE if t is None else (t.data_ptr(), t.stride(0), t.stride(1))
    address = lambda t: 0 if t is None else t.data_ptr()
    out = _pack_grads(*rows, ddecay.data_ptr(), address(drb), address(dib), _param(dh0, dims[1:], "dh0", at))
    _ws, ws, nbytes = _opaque(workspace, _lib.bppsa_gated_scan_backward_workspace_bytes(*dims), at)
    _check(_lib.bppsa_gated_scan_backward(layer, _pack_rows(*_rows(dy, x.shape, x.dtype, "dy", at)),
                                          _param(dh_last, dims[1:], "dh_last", at), _states(states, dims, at), out, ws, nbytes,
                                          _here(at)), "bppsa_gated_scan_backward")
    dx, dr, di, dz = made
    return GatedGrads(dx, dr, di, ddecay, dz, drb, dib, dh0)


def gated_scan_step(x, r, i, decay, state, z=None, r_bias=None, i_bias=None, slots=None, y=None, stream=None):
    """bppsa_gated_scan_step: y [B, D] of one token of each stream; state [slots, D] float32 is advanced in place.

    x, r, i, z [B, D]; slots [B] int32, a row with one outside the state (-1, say) belongs to no stream."""
    if stream is not None:
        return _aside(stream, gated_scan_step, x, r, i, decay, state, z, r_bias, i_bias, slots, y)
    layer, (_, B, D), at = _layer(True, x, r, i, decay, z, r_bias, i_bias)
    states = _whole(state, _f32, "state", at)
    slots_in_state = state.shape[0]
    if state.shape != (slots_in_state, D):
        raise ValueError("state must be [slots, %d], got %s" % (D, tuple(state.shape)))
    y, out = _token_output(y, x, at)
    _check(_lib.bppsa_gated_scan_step(layer, out, states, slots_in_state, _slots(slots, B, slots_in_state, at), _here(at)),
           "bppsa_gated_scan_step")
    return y
