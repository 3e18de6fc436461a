"""ctypes binding of the optimiser over many tensors (bppsa_adamw_step in include/bppsa.h)."""
from __future__ import annotations

import ctypes
import struct

import torch

from .binding import _check, _lib, _ptr, _stream

BLOCK = 256                        # BPPSA_ADAMW_BLOCK
_ROW = 9                           # words of a bppsa_adamw_tensor, the second the gradient's address
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_f32 = torch.float32

_c_int, _c_void_p, _c_double, _c_int64 = ctypes.c_int, ctypes.c_void_p, ctypes.c_double, ctypes.c_int64
_lib.bppsa_adamw_pieces.restype = _c_int64
_lib.bppsa_adamw_pieces.argtypes = [_c_int, _c_void_p, _c_void_p]
_lib.bppsa_adamw_step.restype = _c_int
_lib.bppsa_adamw_step.argtypes = [_c_int, _c_void_p, _c_int64, _c_void_p, _c_int, _c_int, _c_int] + [_c_double] * 4 + \
    [ctypes.c_uint32, _c_void_p]


class AdamW:
    """AdamW over many tensors by one launch a step, with the moments in 32 bits or in 8.

    params: contiguous float32 tensors, updated in place; grads: their gradients, contiguous, all of one type (float32,
    bfloat16 or float16), read where they are at every step; copies: bfloat16 tensors that receive the new parameters, or
    None.  weight_decay: one number or one for each tensor.  `state` (made here unless given) is a dict of lists, a tensor for
    each parameter: "m" and "v", float32; with state_bits=8 float8_e4m3fn, with "m_scale" and "v_scale", float32 of one value
    for each 256, and "v" then stands for the root of the second moment.  The tensors' addresses are taken once, here: replace
    their values, not the tensors, but for gradients that a program makes anew, see read_gradients().  `t` counts the steps;
    lr, beta1, beta2 and eps are read at every step."""

    def __init__(self, params, grads, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, copies=None,
                 state=None):
        params, grads = list(params), list(grads)
        if not params or len(params) != len(grads):
            raise ValueError("AdamW needs as many gradients as parameters, and one at least")
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8, got %r" % (state_bits,))
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(params)
        if len(decay) != len(params) or (copies is not None and len(copies) != len(params)):
            raise ValueError("weight_decay and copies need one entry for each parameter")
        if not isinstance(params[0], torch.Tensor):
            raise ValueError("parameters must be float32 tensors")
        if not isinstance(grads[0], torch.Tensor) or grads[0].dtype not in _TYPES:
            raise ValueError("gradients must be float32, bfloat16 or float16 tensors")
        self.params, self.grads, self.copies = params, grads, None if copies is None else list(copies)
        self.state_bits, self.lr, self.beta1, self.beta2, self.eps, self.t = state_bits, lr, beta1, beta2, eps, 0
        kind = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        names = {"m": kind, "v": kind}
        if state_bits == 8:
            names.update(m_scale=torch.float32, v_scale=torch.float32)
        size = lambda p, name: -(-p.numel() // BLOCK) if name.endswith("scale") else p.numel()
        if state is None:
            make = lambda p, name, t: torch.zeros(size(p, name), dtype=torch.uint8 if t is torch.float8_e4m3fn else t,
                                                  device=p.device).view(t)
            state = {name: [make(p, name, t) for p in params] for name, t in names.items()}
        if set(state) != set(names) or any(len(x) != len(params) for x in state.values()):
            raise ValueError("state must hold %s for each parameter" % ", ".join(names))
        self.state = {name: list(x) for name, x in state.items()}
        device, self._grad_type, rows, lengths = params[0].device, _TYPES[grads[0].dtype], [], []
        self._device = device.index
        kinds = [("params", params, _f32), ("grads", grads, grads[0].dtype)] + [("state[%r]" % name, self.state[name], t) for name, t in names.items()]
        if copies is not None:
            kinds.append(("copies", self.copies, torch.bfloat16))
        pack, blank = struct.Struct("@7Pqd").pack, () if state_bits == 8 else (0, 0)
        for k, p in enumerate(params):
            n = p.numel() if isinstance(p, torch.Tensor) else 0
            counts = (n, n, n, n, -(-n // BLOCK), -(-n // BLOCK), n) if state_bits == 8 else (n, n, n, n, n)
            at = []
            for (name, of, t), count in zip(kinds, counts):
                x = of[k]
                if type(x) is not torch.Tensor or x.dtype is not t or not x.is_cuda or not x.is_contiguous():
                    _ptr(x, t, "%s[%d]" % (name, k))       # says what is wrong, if anything is
                if x is None or x.numel() != count or x.device != device:
                    raise ValueError("%s[%d] must have %d values on %s" % (name, k, count, device))
                at.append(x.data_ptr())
            copy = at.pop() if copies is not None else 0
            rows.append(pack(*at, *blank, copy, n, float(decay[k])))
            lengths.append(n)
        n = (ctypes.c_int64 * len(params))(*lengths)
        self._n_pieces = int(_lib.bppsa_adamw_pieces(len(params), n, None))
        if self._n_pieces < 1:
            raise ValueError("AdamW: nothing to update")
        self._table = bytearray(b"".join(rows))              # what the device has a copy of
        pieces = torch.empty((self._n_pieces, 2), dtype=torch.int32)
        _lib.bppsa_adamw_pieces(len(params), n, pieces.data_ptr())
        self._pieces = pieces.to(device)
        self._tensors = torch.frombuffer(self._table, dtype=torch.uint8).to(device)
        # the streams that what lasts is kept for, and the table with its gradients
        self._streams, self._readers = ({torch.cuda.current_stream(device).cuda_stream} for _ in range(2))

    def read_gradients(self, grads):
        """Reads the gradients from these tensors from now on, of the sizes and the type of those before."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("AdamW needs as many gradients as parameters")
        kind, device, at = self.grads[0].dtype, self.params[0].device, []
        for k, (g, p) in enumerate(zip(grads, self.params)):
            where = _ptr(g, kind, "grads[%d]" % k)
            if where is None or g.numel() != p.numel() or g.device != device:
                raise ValueError("grads[%d] must have %d values on %s" % (k, p.numel(), device))
            at.append(where)
        table = memoryview(self._table).cast("q")
        table[1::_ROW] = memoryview(bytearray(struct.pack("@%dq" % len(at), *at))).cast("q")
        self.grads = grads
        self._tensors = torch.frombuffer(self._table, dtype=torch.uint8).to(device)
        self._readers = {torch.cuda.current_stream(device).cuda_stream}

    def _keep(self, on, stream):
        """For a stream that steps run on: the optimiser may go before it is done, and read_gradients() lets the table go."""
        for kept, held in ((self._streams, (self._pieces, *self.params, *(self.copies or ()), *sum(self.state.values(), []))),
                           (self._readers, (self._tensors, *self.grads))):
            if on not in kept:
                kept.add(on)
                for x in held:
                    x.record_stream(stream)

    def step(self, seed=None, stream=None):
        """One update.  With 8-bit moments `seed` (the number of the step unless given) decides which values that are
        rounded by chance go up."""
        t = self.t + 1
        seed = t if seed is None else int(seed)
        now = torch.cuda.current_device() if stream is None else stream.device.index
        if now != self._device:
            raise ValueError("AdamW: the tensors are on cuda:%d, the stream is cuda:%d's" % (self._device, now))
        on = _stream(stream)
        if on not in self._streams or on not in self._readers:
            self._keep(on, torch.cuda.current_stream() if stream is None else stream)
        _check(_lib.bppsa_adamw_step(len(self.params), self._tensors.data_ptr(), self._n_pieces, self._pieces.data_ptr(),
                                     self._grad_type, self.state_bits, t, self.lr, self.beta1, self.beta2, self.eps,
                                     seed & 0xFFFFFFFF, on), "bppsa_adamw_step")
        self.t = t
