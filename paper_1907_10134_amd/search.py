"""ctypes binding of a beam search's step: the selection over beams and vocabulary, and the move of the beams' states between
slots (bppsa_beam_select and bppsa_beam_move in include/bppsa.h)."""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple

import torch

from .binding import _aside, _check, _lib
from .ssm import _TYPES, _f32, _here, _i32, _on, _opaque, _param, _whole

_c_int, _c_void_p, _c_size_t, _c_int64 = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
for _name, _res, _args in (
        ("bppsa_beam_select_workspace_bytes", _c_size_t, [_c_int] * 3),
        ("bppsa_beam_select", _c_int, [_c_void_p] * 3 + [_c_size_t, _c_void_p]),
        ("bppsa_beam_pieces", _c_int64, [_c_int, _c_void_p, _c_void_p]),
        ("bppsa_beam_move", _c_int, [_c_void_p, _c_int64, _c_void_p, _c_int, _c_void_p, _c_void_p, _c_int, _c_void_p])):
    getattr(_lib, _name).restype = _res
    getattr(_lib, _name).argtypes = _args

_pack_beam = struct.Struct("@5iPqqPPP").pack
_pack_choice = struct.Struct("@6P").pack

BeamChoice = namedtuple("BeamChoice", "scores parents tokens finished slots sources")


def beam_select_workspace_bytes(B, W, V):
    return int(_lib.bppsa_beam_select_workspace_bytes(B, W, V))


def beam_select(logits, scores, finished=None, end=-1, slots=None, workspace=None, stream=None):
    """bppsa_beam_select: the W best continuations of W beams for each of B sequences, best first, as BeamChoice.

    logits [B, W, V] float32, bfloat16 or float16, the V logits side by side; scores [B, W] float32, minus infinity for beams
    that there are not (yet); finished [B, W] bool: these beams go on with the token `end` alone, at their score; slots
    [B, W] int32: where the beams keep their states.  Of the result, finished is None without `end`, and slots and sources
    without slots: BeamStates.move(sources, slots) brings the states of the beams that have several children to all of them."""
    if stream is not None:
        return _aside(stream, beam_select, logits, scores, finished, end, slots, workspace)
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a torch.Tensor")
    t, at = logits.dtype, logits.get_device()
    _on(logits, at, "logits")
    if logits.dim() != 3:
        raise ValueError("logits must be [B, W, V]")
    if t not in _TYPES:
        raise ValueError("logits must be float32, bfloat16 or float16, got %s" % t)
    B, W, V = logits.shape
    sb, sw, sv = logits.stride()
    if sv != 1 and V > 1:
        raise ValueError("logits must be contiguous in the vocabulary")
    if scores is None:
        raise TypeError("scores must be a torch.Tensor")
    shape = (B, W)
    if finished is not None and not 0 <= end < V:
        raise ValueError("beam_select: finished needs an end within the vocabulary, got %r" % (end,))
    if not -1 <= end < V:
        raise ValueError("end must be a token or -1, got %r" % (end,))
    packed = _pack_beam(B, W, V, _TYPES[t], end, logits.data_ptr(), sb, sw, _param(scores, shape, "scores", at),
                        _param(finished, shape, "finished", at, torch.bool), _param(slots, shape, "slots", at, _i32))
    # the results of four bytes as rows of one array: one allocation instead of five
    made = torch.empty((3 if slots is None else 5, B, W), dtype=_i32, device=logits.device).unbind(0)
    c = BeamChoice(made[0].view(_f32), made[1], made[2], None if end < 0 else torch.empty(shape, dtype=torch.bool, device=logits.device),
                   *((None, None) if slots is None else made[3:]))
    _ws, ws, nbytes = _opaque(workspace, _lib.bppsa_beam_select_workspace_bytes(B, W, V), at)
    _check(_lib.bppsa_beam_select(packed, _pack_choice(*(0 if x is None else x.data_ptr() for x in c)), ws, nbytes, _here(at)),
           "bppsa_beam_select")
    return c


class BeamStates:
    """States of many kinds, each a contiguous tensor [slots, ...] of any type, that move together by one launch.

    The tensors' addresses are taken once, here: replace their values, not the tensors.  A captured graph reads this object's lists
    at every replay: the object has to live as long as the graph."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        if not self.tensors or not all(isinstance(x, torch.Tensor) for x in self.tensors):
            raise TypeError("BeamStates needs torch.Tensors, one at least")
        first = self.tensors[0]
        self._device = first.get_device()
        rows, sizes = [], []
        for k, x in enumerate(self.tensors):
            _on(x, self._device, "tensors[%d]" % k)
            if x.dim() < 1 or x.shape[0] != first.shape[0] or x.numel() == 0:
                raise ValueError("tensors[%d] must be [%s, ...] and not empty, got %s" % (k, first.shape[0] if first.dim() else "slots", tuple(x.shape)))
            if not x.is_contiguous():
                raise ValueError("tensors[%d] must be contiguous" % k)
            sizes.append(x.numel() // x.shape[0] * x.element_size())
            rows.append(struct.pack("@Pq", x.data_ptr(), sizes[-1]))
        self.slots = first.shape[0]
        n = (_c_int64 * len(sizes))(*sizes)
        self._n_pieces = int(_lib.bppsa_beam_pieces(len(sizes), n, None))
        if self._n_pieces < 1:
            raise ValueError("BeamStates: a slot's states are too large")
        # the table of tensors and the list of pieces behind it, in one copy
        both = torch.empty(16 * len(rows) + 8 * self._n_pieces, dtype=torch.uint8)
        ctypes.memmove(both.data_ptr(), b"".join(rows), 16 * len(rows))
        _lib.bppsa_beam_pieces(len(sizes), n, both.data_ptr() + 16 * len(rows))
        self._streams = {torch.cuda.current_stream(first.device).cuda_stream}      # that the lists are kept for
        self._lists = both.to(first.device)
        self._table = self._lists.data_ptr()
        self._pieces = self._table + 16 * len(rows)

    def move(self, sources, slots, stream=None):
        """bppsa_beam_move: copies the states of slot sources[...] to slot slots[...], int32 of the same shape; a source of -1 is
        none.  No slot may be written twice, or read and written."""
        if stream is not None:
            _aside(stream, self._move, sources, slots)
        else:
            self._move(sources, slots)

    def _move(self, sources, slots):
        if not isinstance(slots, torch.Tensor):
            raise TypeError("slots must be a torch.Tensor")
        if sources is None:
            raise TypeError("sources must be a torch.Tensor")
        to, of = _whole(slots, _i32, "slots", self._device), _param(sources, slots.shape, "sources", self._device, _i32)
        stream = _here(self._device)
        if stream not in self._streams:            # the object may go before that stream has read what only it keeps
            self._streams.add(stream)
            for x in (self._lists, *self.tensors):
                x.record_stream(torch.cuda.current_stream())
        _check(_lib.bppsa_beam_move(self._table, self._n_pieces, self._pieces, slots.numel(), of, to, self.slots, stream), "bppsa_beam_move")
