"""What stands between an expert's two products in training: gated activations with dropout, and their gradient, on torch tensors.

    h = activate(up_rows, act="silu", p=0.1, seed=seed, offsets=r.offsets)   # rows in expert order: act(gate) * other, dropped out

Dropout's mask comes from a counter-based generator (Philox-4x32-10) and is never stored: the gradient forms it again from the same seed. ``seed`` is a tensor of two int64 on the
device, the generator's key and the number of the call, so that a captured step draws other masks when its contents change. Streams and
errors are those of experts.py; the operators are the C calls ``hccl_activate`` and ``hccl_activate_backward``.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as hb
from .experts import _cols, _dtype, _matrix, _new, _on, _refuse, _same_type, _stream, _vector

_activate, _activate_backward = hb.packed("hccl_activate"), hb.packed("hccl_activate_backward")
ACTS = {"silu": hb.ACT_SILU, "gelu": hb.ACT_GELU, "relu": hb.ACT_RELU}


def _config(x, act, gated, p, seed, offsets):
    """The call's leading arguments, the width of the result, and the end of the rows that count."""
    a = ACTS.get(act)
    if a is None:
        _refuse(hb.ERR_INVALID_ARG, "act %r, expected one of %s" % (act, ", ".join(ACTS)))
    if not isinstance(p, (int, float)) or not 0 <= p < 1:
        _refuse(hb.ERR_INVALID_ARG, "p = %r must be at least 0 and below 1" % (p,))
    ldx, dt, dev = _matrix(x, "x"), _dtype(x, "x"), x.get_device()
    I = x.shape[1]
    if gated:
        if I % 2:
            _refuse(hb.ERR_COUNT_MISMATCH, "x has %d columns, a gated activation takes two halves" % I)
        I //= 2
    at = 0
    if p > 0:
        if seed is None:
            _refuse(hb.ERR_INVALID_ARG, "dropout needs a seed: two int64 on the device")
        _vector(seed, "seed", torch.int64, 2, dev)
        at = seed.data_ptr()
    end, groups = 0, 0
    if offsets is not None:
        groups = offsets.numel() - 1
        if groups < 1:
            _refuse(hb.ERR_COUNT_MISMATCH, "offsets has %d elements, expected one more than there are experts" % offsets.numel())
        _vector(offsets, "offsets", torch.int32, groups + 1, dev)
        end = offsets.data_ptr()
    return (a, 1 if gated else 0, struct.unpack("<q", struct.pack("<d", p))[0], at), ldx, dt, dev, I, end, groups


def _forward(x, act, gated, p, seed, offsets, out):
    head, ldx, dt, dev, I, end, groups = _config(x, act, gated, p, seed, offsets)
    out, ldy = _new(out, x.shape[0], I, x, "out", dev)
    _on(dev, _activate)(*head, x.data_ptr(), ldx, x.shape[0], I, dt, end, groups, out.data_ptr(), ldy, _stream(dev))
    return out


def activate(x: torch.Tensor, act: str = "silu", gated: bool = True, p: float = 0.0, seed: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """gated: x [M, 2 I], the gate's half first, result act(gate) * other [M, I]; otherwise act(x). Each element is dropped with probability p, the others grow by
    1 / (1 - p). offsets (int32 [experts + 1]): rows from offsets[-1] on are not read and become 0. act: "silu", "gelu" (by the normal distribution), "relu"."""
    if x.requires_grad and torch.is_grad_enabled():
        if out is not None:
            _refuse(hb.ERR_INVALID_ARG, "activate: out= cannot carry a gradient")
        return _Activate.apply(x, act, gated, p, seed, offsets)
    return _forward(x, act, gated, p, seed, offsets, out)


def activate_backward(dy: torch.Tensor, x: torch.Tensor, act: str = "silu", gated: bool = True, p: float = 0.0, seed: Optional[torch.Tensor] = None,
                      offsets: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of x for a gradient dy of activate's result; rows from offsets[-1] on become 0."""
    head, ldx, dt, dev, I, end, groups = _config(x, act, gated, p, seed, offsets)
    ldy = _matrix(dy, "dy", I, x.shape[0], dev)
    _same_type(dy, x, "activate backward")
    out, ldd = _new(out, x.shape[0], x.shape[1], x, "dx", dev)
    _on(dev, _activate_backward)(*head, dy.data_ptr(), ldy, x.data_ptr(), ldx, x.shape[0], I, dt, end, groups, out.data_ptr(), ldd, _stream(dev))
    return out


class _Activate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, act, gated, p, seed, offsets):
        ctx.save_for_backward(x, seed if p else None, offsets)  # a seed that was written to since has no gradient to give
        ctx.config = (act, gated, p)
        return _forward(x, act, gated, p, seed, offsets, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, seed, offsets = ctx.saved_tensors
        act, gated, p = ctx.config
        return activate_backward(_cols(dy), x, act, gated, p, seed, offsets), None, None, None, None, None
