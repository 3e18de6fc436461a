"""ctypes binding of the selective state space layer: the scan, the short convolution in front of it, their gradients and
their steps for single tokens, with the names of the C ABI in include/bppsa.h.

Activations are float32, bfloat16 or float16, all of one call the same, [T, B, channels] with the channels contiguous and any
strides of time and sample; parameters, states and their gradients are contiguous float32.  A call runs on the current stream
or on `stream`; the caller orders that stream with the ones that make the inputs and use the results.
"""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple

import torch

from .binding import _aside, _check, _lib, _ptr, _raw_stream, _workspace

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_i32, _f32, _plain = torch.int32, torch.float32, torch.contiguous_format

_c_int, _c_void_p, _c_size_t = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
for _name, _res, _args in (
        ("bppsa_ssm_scan_states_bytes", _c_size_t, [_c_int] * 4),
        ("bppsa_ssm_scan_workspace_bytes", _c_size_t, [_c_int] * 5),
        ("bppsa_ssm_scan", _c_int, [_c_void_p] * 5 + [_c_size_t, _c_void_p]),
        ("bppsa_ssm_scan_backward_workspace_bytes", _c_size_t, [_c_int] * 5),
        ("bppsa_ssm_scan_backward", _c_int, [_c_void_p] * 5 + [_c_size_t, _c_void_p]),
        ("bppsa_ssm_scan_step", _c_int, [_c_void_p] * 3 + [_c_int] + [_c_void_p] * 2),
        ("bppsa_ssm_conv", _c_int, [_c_void_p] * 4),
        ("bppsa_ssm_conv_backward_workspace_bytes", _c_size_t, [_c_int] * 4),
        ("bppsa_ssm_conv_backward", _c_int, [_c_void_p] * 7 + [_c_size_t, _c_void_p]),
        ("bppsa_ssm_conv_step", _c_int, [_c_void_p] * 3 + [_c_int] + [_c_void_p] * 2)):
    getattr(_lib, _name).restype = _res
    getattr(_lib, _name).argtypes = _args

# The C structs as bytes: a struct module's pack takes 1 us where a ctypes Structure of as many fields takes 6.
_pack_rows = struct.Struct("@Pqq").pack
_pack_layer = struct.Struct("@6i" + "Pqq" * 5 + "P" * 5).pack
_pack_grads = struct.Struct("@" + "Pqq" * 3 + "P" * 6).pack
_pack_conv = struct.Struct("@6iPqq" + "P" * 4).pack


def _on(t, device, name):
    """Refuses what is no tensor on the GPU, or on another one than the first argument."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if t.get_device() != device:
        raise ValueError("%s must be on cuda:%d like the first argument, not on %s" % (name, device, t.device))


def _rows(t, shape, dtype, name, device, groups=False):
    """(pointer, time stride, sample stride) of an activation [T, B, channels] or [T, B, G, N]."""
    _on(t, device, name)
    if t.dtype is not dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    s = t.stride()
    if groups:
        if (s[-1] != 1 and shape[-1] > 1) or (s[-2] != shape[-1] and shape[-2] > 1):
            raise ValueError("%s must be contiguous in its last two dimensions" % name)
    elif s[-1] != 1 and shape[-1] > 1:
        raise ValueError("%s must be contiguous in its channels" % name)
    return t.data_ptr(), s[0], s[1]


def _token(t, shape, dtype, name, device):
    """The same of one token of each stream, [B, channels]: (pointer, 0, sample stride)."""
    if type(t) is torch.Tensor and t.dtype is dtype and t.get_device() == device and t.shape == shape:
        s = t.stride()
        if s[1] == 1 or shape[1] == 1:
            return t.data_ptr(), 0, s[0]
    p, _, b = _rows(t.unsqueeze(0) if isinstance(t, torch.Tensor) else t, (1,) + tuple(shape), dtype, name, device)   # names what is wrong
    return p, 0, b


def _param(t, shape, name, device, dtype=torch.float32):
    if t is None:
        return 0
    if type(t) is torch.Tensor and t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    _on(t, device, name)
    p = _ptr(t, dtype, name)
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return p


def _whole(t, dtype, name, device):
    """The address of a contiguous array whose shape the caller looks at."""
    if type(t) is torch.Tensor and t.dtype is dtype and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    _on(t, device, name)
    return _ptr(t, dtype, name)


_NONE = (0, 0, 0)


def _own(t, shape, device):
    """The address of an optional fp32 parameter if it is what it has to be, None if that has to be looked at closer."""
    if t is None:
        return 0
    if t.dtype is _f32 and t.get_device() == device and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    return None


def _quick_layer(token, u, dt, A, Bm, Cm, skip, z, dt_bias, h0, lengths):
    """_layer in one go where every tensor is as it should be with nothing odd about it (6 us instead of 11); None otherwise."""
    try:
        t, wide, narrow, at = u.dtype, u.shape, Bm.shape, u.get_device()
        if token:
            (B, D), T, (_, G, N) = wide, 1, narrow
        else:
            (T, B, D), (_, _, G, N) = wide, narrow
        if not (dt.dtype is t and Bm.dtype is t and Cm.dtype is t and A.dtype is _f32 and dt.shape == wide and Cm.shape == narrow and
                narrow[:-2] == wide[:-1] and A.shape == (D, N) and
                at >= 0 and dt.get_device() == at and Bm.get_device() == at and Cm.get_device() == at and
                A.get_device() == at and A.is_contiguous()):
            return None
        su, sd, sb, sc = u.stride(), dt.stride(), Bm.stride(), Cm.stride()
        if not (su[-1] == sd[-1] == sb[-1] == sc[-1] == 1 and sb[-2] == sc[-2] == N):
            return None
        pz, sz = 0, su
        if z is not None:
            sz = z.stride()
            if not (z.dtype is t and z.get_device() == at and z.shape == wide and sz[-1] == 1):
                return None
            pz = z.data_ptr()
        params = (A.data_ptr(), _own(skip, (D,), at), _own(dt_bias, (D,), at), _own(h0, (B, D, N), at))
        if None in params:
            return None
        ends = 0 if lengths is None else _param(lengths, (B,), "lengths", at, _i32)
        kind = _TYPES[t]
        if token:
            return _pack_layer(1, B, D, N, G, kind, u.data_ptr(), 0, su[0], dt.data_ptr(), 0, sd[0], pz, 0, sz[0], Bm.data_ptr(), 0,
                               sb[0], Cm.data_ptr(), 0, sc[0], *params, ends), (1, B, D, N, G), at
        return _pack_layer(T, B, D, N, G, kind, u.data_ptr(), su[0], su[1], dt.data_ptr(), sd[0], sd[1], pz, sz[0], sz[1],
                           Bm.data_ptr(), sb[0], sb[1], Cm.data_ptr(), sc[0], sc[1], *params, ends), (T, B, D, N, G), at
    except (AttributeError, KeyError, TypeError, ValueError):
        return None


def _layer(token, u, dt, A, Bm, Cm, skip, z, dt_bias, h0=None, lengths=None):
    """The bytes of bppsa_ssm, (T, B, D, N, G) and the device's number; token: of [B, channels], T = 1."""
    quick = _quick_layer(token, u, dt, A, Bm, Cm, skip, z, dt_bias, h0, lengths)
    if quick is not None:
        return quick
    if not (isinstance(u, torch.Tensor) and isinstance(Bm, torch.Tensor)):
        raise TypeError("u and Bm must be torch.Tensors")
    if token:
        if u.dim() != 2 or Bm.dim() != 3:
            raise ValueError("u must be [B, D] and Bm [B, G, N]")
        one = lambda t: t.unsqueeze(0) if isinstance(t, torch.Tensor) else t
        return _layer(False, one(u), one(dt), A, one(Bm), one(Cm), skip, one(z), dt_bias)
    if u.dim() != 3 or Bm.dim() != 4:
        raise ValueError("u must be [T, B, D] and Bm [T, B, G, N]")
    T, B, D = u.shape
    G, N = Bm.shape[2], Bm.shape[3]
    t, wide, narrow, at = u.dtype, u.shape, (T, B, G, N), u.get_device()
    if t not in _TYPES:
        raise ValueError("activations must be float32, bfloat16 or float16, got %s" % t)
    if A is None:
        raise TypeError("A must be a torch.Tensor")
    return _pack_layer(T, B, D, N, G, _TYPES[t], *_rows(u, wide, t, "u", at), *_rows(dt, wide, t, "dt", at),
                       *(_NONE if z is None else _rows(z, wide, t, "z", at)), *_rows(Bm, narrow, t, "Bm", at, True),
                       *_rows(Cm, narrow, t, "Cm", at, True), _param(A, (D, N), "A", at), _param(skip, (D,), "skip", at),
                       _param(dt_bias, (D,), "dt_bias", at), _param(h0, (B, D, N), "h0", at),
                       _param(lengths, (B,), "lengths", at, _i32)), (T, B, D, N, G), at


# without what torch.cuda.current_device does for a program that has not used the GPU yet
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _like(t):
    """A new array of t's shape and order of dimensions, its channels side by side also where t is windows of one array, whose order
    torch cannot tell."""
    new = torch.empty_like(t)
    return new if new.stride(-1) == 1 else torch.empty_like(t, memory_format=_plain)


def _output(y, x, name, device):
    """(the array, the bytes of bppsa_rows) of an output like x [T, B, D], made here unless given."""
    if y is None:
        y = torch.empty_like(x)
        s = y.stride()
        if s[2] == 1:
            return y, _pack_rows(y.data_ptr(), s[0], s[1])
        y = torch.empty_like(x, memory_format=_plain)          # see _like
    return y, _pack_rows(*_rows(y, x.shape, x.dtype, name, device))


def _token_output(y, x, device):
    """The same of one token of each stream, like x [B, D]."""
    if y is None:
        y = torch.empty_like(x)
        s = y.stride()
        if s[1] == 1:
            return y, _pack_rows(y.data_ptr(), 0, s[0])
        y = torch.empty_like(x, memory_format=_plain)
    return y, _pack_rows(*_token(y, x.shape, x.dtype, "y", device))


def _here(device):
    """The current stream, which has to be one of the tensors' device: a kernel started elsewhere would use them from there."""
    now = _current_device()
    if now != device:
        raise ValueError("the tensors are on cuda:%d, the current device is cuda:%d" % (device, now))
    return _raw_stream(now) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _opaque(workspace, nbytes, device):
    """(tensor that has to live through the call, pointer, bytes) of a scratch array."""
    if workspace is None:
        if not nbytes:
            return None, None, 0
        workspace = _workspace(nbytes, device)
    else:
        _on(workspace, device, "workspace")
        _ptr(workspace, workspace.dtype, "workspace")          # contiguous
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def ssm_scan_workspace_bytes(T, B, D, N, G):
    return int(_lib.bppsa_ssm_scan_workspace_bytes(T, B, D, N, G))


def ssm_scan_states(T, B, D, N, device="cuda"):
    """The array that ssm_scan(states=) fills for ssm_scan_backward: bppsa_ssm_scan_states_bytes(T, B, D, N) bytes."""
    n = int(_lib.bppsa_ssm_scan_states_bytes(T, B, D, N))
    if not n:
        raise ValueError("ssm_scan_states: no such sizes (%d, %d, %d, %d)" % (T, B, D, N))
    return torch.empty(n, dtype=torch.uint8, device=device)


def _states(states, dims, device):
    if states is None:
        return None
    at = _whole(states, torch.uint8, "states", device)
    if states.numel() < _lib.bppsa_ssm_scan_states_bytes(*dims[:4]):
        raise ValueError("states is too small for these sizes")
    return at


def ssm_scan(u, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, h0=None, lengths=None, y=None, h_last=None, states=None,
             workspace=None, stream=None):
    """bppsa_ssm_scan: y [T, B, D] of the selective scan of u under steps softplus(dt + dt_bias).

    u, dt, z [T, B, D]; Bm, Cm [T, B, G, N]; A [D, N]; skip, dt_bias [D]; h0 [B, D, N]; lengths [B] int32.  h_last [B, D, N]
    receives the last states, states (see ssm_scan_states) what ssm_scan_backward needs."""
    if stream is not None:
        return _aside(stream, ssm_scan, u, dt, A, Bm, Cm, skip, z, dt_bias, h0, lengths, y, h_last, states, workspace)
    layer, dims, at = _layer(False, u, dt, A, Bm, Cm, skip, z, dt_bias, h0, lengths)
    T, B, D, N, G = dims
    y, out = _output(y, u, "y", at)
    _ws, ws, nbytes = _opaque(workspace, _lib.bppsa_ssm_scan_workspace_bytes(T, B, D, N, G), at)
    _check(_lib.bppsa_ssm_scan(layer, out, _param(h_last, (B, D, N), "h_last", at),
                               _states(states, dims, at), ws, nbytes, _here(at)), "bppsa_ssm_scan")
    return y


SsmGrads = namedtuple("SsmGrads", "du ddt dA dBm dCm dskip dz ddt_bias dh0")


def ssm_scan_backward_workspace_bytes(T, B, D, N, G):
    return int(_lib.bppsa_ssm_scan_backward_workspace_bytes(T, B, D, N, G))


def ssm_scan_backward(dy, u, dt, A, Bm, Cm, states, skip=None, z=None, dt_bias=None, h0=None, lengths=None, dh0=None,
                      workspace=None, stream=None):
    """bppsa_ssm_scan_backward: the gradients of sum(y dy), as SsmGrads; the other arguments are those of the ssm_scan call
    that filled `states`.  dskip, dz and ddt_bias are None where there is no such input; dh0 [B, D, N] is filled if given."""
    if stream is not None:
        return _aside(stream, ssm_scan_backward, dy, u, dt, A, Bm, Cm, states, skip, z, dt_bias, h0, lengths, dh0, workspace)
    layer, dims, at = _layer(False, u, dt, A, Bm, Cm, skip, z, dt_bias, h0, lengths)
    T, B, D, N, G = dims
    if states is None:
        raise TypeError("states must be the array that ssm_scan filled")
    t, like = u.dtype, torch.empty_like
    du, ddt = _like(u), _like(dt)
    dz = None if z is None else like(du)
    dBm, dCm = like(Bm, memory_format=_plain), like(Cm, memory_format=_plain)
    dA, dskip, dbias = like(A), None if skip is None else like(skip), None if dt_bias is None else like(dt_bias)
    su, sd = du.stride(), ddt.stride()
    out = _pack_grads(du.data_ptr(), su[0], su[1], ddt.data_ptr(), sd[0], sd[1], 0 if dz is None else dz.data_ptr(), su[0], su[1],
                      dBm.data_ptr(), dCm.data_ptr(), dA.data_ptr(), 0 if dskip is None else dskip.data_ptr(),
                      0 if dbias is None else dbias.data_ptr(), _param(dh0, (B, D, N), "dh0", at))
    _ws, ws, nbytes = _opaque(workspace, _lib.bppsa_ssm_scan_backward_workspace_bytes(T, B, D, N, G), at)
    _check(_lib.bppsa_ssm_scan_backward(layer, _pack_rows(*_rows(dy, u.shape, t, "dy", at)), _states(states, dims, at), out, ws,
                                        nbytes, _here(at)), "bppsa_ssm_scan_backward")
    return SsmGrads(du, ddt, dA, dBm, dCm, dskip, dz, dbias, dh0)


def _slots(slots, B, slots_in_state, device):
    if slots is None:
        if slots_in_state < B:
            raise ValueError("state has fewer slots than the batch has rows")
        return None
    return _param(slots, (B,), "slots", device, _i32)


def ssm_scan_step(u, dt, A, Bm, Cm, state, skip=None, z=None, dt_bias=None, slots=None, y=None, stream=None):
    """bppsa_ssm_scan_step: y [B, D] of one token of each stream; state [slots, D, N] float32 is advanced in place.

    u, dt, z [B, D]; Bm, Cm [B, G, N]; slots [B] int32, a row with one outside the state (-1, say) belongs to no stream."""
    if stream is not None:
        return _aside(stream, ssm_scan_step, u, dt, A, Bm, Cm, state, skip, z, dt_bias, slots, y)
    layer, (_, B, D, N, _), at = _quick_layer(True, u, dt, A, Bm, Cm, skip, z, dt_bias, None, None) or \
        _layer(True, u, dt, A, Bm, Cm, skip, z, dt_bias)
    states = _whole(state, _f32, "state", at)
    slots_in_state = state.shape[0]
    if state.shape != (slots_in_state, D, N):
        raise ValueError("state must be [slots, %d, %d], got %s" % (D, N, tuple(state.shape)))
    y, out = _token_output(y, u, at)
    _check(_lib.bppsa_ssm_scan_step(layer, out, states, slots_in_state, _slots(slots, B, slots_in_state, at), _here(at)),
           "bppsa_ssm_scan_step")
    return y


def _conv(x, weight, bias, silu, state0, lengths):
    if not (isinstance(x, torch.Tensor) and isinstance(weight, torch.Tensor)):
        raise TypeError("x and weight must be torch.Tensors")
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x must be [T, B, D] and weight [D, W]")
    T, B, D = x.shape
    W, at = weight.shape[1], x.get_device()
    if x.dtype not in _TYPES:
        raise ValueError("activations must be float32, bfloat16 or float16, got %s" % x.dtype)
    return _pack_conv(T, B, D, W, _TYPES[x.dtype], bool(silu), *_rows(x, x.shape, x.dtype, "x", at),
                      _param(weight, (D, W), "weight", at), _param(bias, (D,), "bias", at),
                      _param(state0, (B, W - 1, D), "state0", at, x.dtype), _param(lengths, (B,), "lengths", at, _i32)), (T, B, D, W), at


def ssm_conv(x, weight, bias=None, silu=True, state0=None, lengths=None, y=None, state_last=None, stream=None):
    """bppsa_ssm_conv: the causal convolution of x [T, B, D] with weight [D, W], channel by channel, and silu.

    state0 [B, W-1, D] holds the inputs in front of the first; state_last, of the same shape, receives the last ones."""
    if stream is not None:
        return _aside(stream, ssm_conv, x, weight, bias, silu, state0, lengths, y, state_last)
    conv, (_, B, D, W), at = _conv(x, weight, bias, silu, state0, lengths)
    y, out = _output(y, x, "y", at)
    _check(_lib.bppsa_ssm_conv(conv, out, _param(state_last, (B, W - 1, D), "state_last", at, x.dtype), _here(at)), "bppsa_ssm_conv")
    return y


SsmConvGrads = namedtuple("SsmConvGrads", "dx dweight dbias dstate0")


def ssm_conv_backward(dy, x, weight, bias=None, silu=True, state0=None, lengths=None, dstate0=None, workspace=None,
                      stream=None):
    """bppsa_ssm_conv_backward: the gradients of sum(y dy), as SsmConvGrads; dstate0 [B, W-1, D] is filled if given."""
    if stream is not None:
        return _aside(stream, ssm_conv_backward, dy, x, weight, bias, silu, state0, lengths, dstate0, workspace)
    conv, (T, B, D, W), at = _conv(x, weight, bias, silu, state0, lengths)
    dx, out = _output(None, x, "dx", at)
    dweight, dbias = torch.empty_like(weight), None if bias is None else torch.empty_like(bias)
    _ws, ws, nbytes = _opaque(workspace, _lib.bppsa_ssm_conv_backward_workspace_bytes(T, B, D, W), at)
    _check(_lib.bppsa_ssm_conv_backward(conv, _pack_rows(*_rows(dy, x.shape, x.dtype, "dy", at)), out, dweight.data_ptr(),
                                        None if dbias is None else dbias.data_ptr(),
                                        _param(dstate0, (B, W - 1, D), "dstate0", at, x.dtype), ws, nbytes, _here(at)),
           "bppsa_ssm_conv_backward")
    return SsmConvGrads(dx, dweight, dbias, dstate0)


def ssm_conv_step(x, weight, bias, state, silu=True, slots=None, y=None, stream=None):
    """bppsa_ssm_conv_step: y [B, D] of one token of each stream; state [slots, W-1, D] is moved on in place."""
    if stream is not None:
        return _aside(stream, ssm_conv_step, x, weight, bias, state, silu, slots, y)
    if not (isinstance(x, torch.Tensor) and isinstance(weight, torch.Tensor)):
        raise TypeError("x and weight must be torch.Tensors")
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x must be [B, D] and weight [D, W]")
    shape, t, at = x.shape, x.dtype, x.get_device()
    B, D = shape
    W = weight.shape[1]
    if t not in _TYPES:
        raise ValueError("activations must be float32, bfloat16 or float16, got %s" % t)
    conv = _pack_conv(1, B, D, W, _TYPES[t], bool(silu), *_token(x, shape, t, "x", at), _param(weight, (D, W), "weight", at),
                      _param(bias, (D,), "bias", at), 0, 0)
    states = _whole(state, t, "state", at)
    slots_in_state = state.shape[0]
    if state.shape != (slots_in_state, W - 1, D):
        raise ValueError("state must be [slots, %d, %d], got %s" % (W - 1, D, tuple(state.shape)))
    y, out = _token_output(y, x, at)
    _check(_lib.bppsa_ssm_conv_step(conv, out, states, slots_in_state, _slots(slots, B, slots_in_state, at), _here(at)),
           "bppsa_ssm_conv_step")
    return y
