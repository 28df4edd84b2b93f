"""Experts in 4-bit floating point on torch tensors: rows in blocks with a scale each, linear layers.

An element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 or its negative, two to a byte, the earlier in the low half. "nvfp4": blocks of 16 with a scale in e4m3 beside
a 32-bit scale for the whole matrix; "mxfp4": blocks of 32 with a power of two, the least with which nothing saturates (OCP's conversion takes half of that where a block's largest is more than
1.5 times a power of two; rows converted so are read the same). The operators are the C calls of include/hccl.h (``hccl_quantize_rows_fp4`` and
the ones after it); streams, scratch and errors are those of experts.py.

    up, down = Fp4Linear.from_float(w_up), Fp4Linear.from_float(w_down)     # [64, inner, hidden], [64, hidden, inner]
    y = up(x, routing=r)                                                    # rows gathered, quantised, multiplied
    rows = quantize_rows(x, routing=r)                                      # in expert order: codes and scales, 0.28 of the bytes that rows in 16 bits have
    h = up.matmul(rows, offsets=r.offsets)
    y = FewTokens(up, down, act="silu")(x, r)                               # a decode step of up to about 8 tokens: the whole layer in two kernels

Codes and scales are two tensors, each of which can be exchanged. The C call takes the distance between rows for both, so that a row's scales may follow its codes in one send buffer; what arrives is
``Fp4Rows`` of two views of the buffer.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from . import binding as hb
from .activation import ACTS
from .experts import (_DT, _dtype, _given, _matrix, _new, _no_gradient, _on, _pad16, _refuse, _scratch, _stream, _vector, Routing)

_quantize, _dequantize = hb.packed("hccl_quantize_rows_fp4"), hb.packed("hccl_dequantize_rows_fp4")
_matmul, _linear, _layer = hb.packed("hccl_matmul_fp4"), hb.packed("hccl_linear_fp4"), hb.packed("hccl_expert_layer_fp4")

FORMATS = {"nvfp4": hb.NVFP4, "mxfp4": hb.MXFP4}
BLOCK = {"nvfp4": 16, "mxfp4": 32}


def _format(name: str) -> int:
    f = FORMATS.get(name)
    if f is None:
        _refuse(hb.ERR_DTYPE, "format %r, expected one of %s" % (name, ", ".join(FORMATS)))
    return f


def _bits(x: float) -> int:
    if x == 1.0:
        return 0x3F800000
    try:
        return struct.unpack("<I", struct.pack("<f", x))[0]
    except (struct.error, OverflowError, TypeError):
        _refuse(hb.ERR_INVALID_ARG, "scale %r is not a 32-bit number" % (x,))


def _wide(scale: float, format: str) -> float:
    if format == "mxfp4":
        return 1.0
    if not isinstance(scale, (int, float)) or not 1e-30 <= scale <= 1e30:
        _refuse(hb.ERR_INVALID_ARG, "scale %r must be a number from 1e-30 to 1e30" % (scale,))
    return float(scale)


def _bytes(t: torch.Tensor, what: str) -> torch.Tensor:
    """Codes or scales, whatever one-byte type they come in."""
    if t.dtype != torch.uint8:
        if t.element_size() != 1 or t.dtype in (torch.int8, torch.bool):
            _refuse(hb.ERR_DTYPE, "%s is %s" % (what, t.dtype))
        t = t.view(torch.uint8)
    return t


class Fp4Rows:
    """Rows in 4 bits: q [rows, (K + 1) // 2] and scale [rows, blocks], both uint8, and the matrix's own scale (1 for "mxfp4")."""

    __slots__ = ("q", "scale", "wide", "format", "K")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, K: int, format: str = "nvfp4", wide: float = 1.0):
        _format(format)
        q, scale = _bytes(q, "q"), _bytes(scale, "scale")
        _matrix(q, "q", (K + 1) // 2)
        _matrix(scale, "scale", (K + BLOCK[format] - 1) // BLOCK[format], q.shape[0], q.get_device())
        self.q, self.scale, self.K, self.format, self.wide = q, scale, K, format, _wide(wide, format)

    def __reduce__(self):
        return Fp4Rows, (self.q, self.scale, self.K, self.format, self.wide)

    @classmethod
    def _made(cls, q, scale, K, format, wide):
        """Of tensors that hold together, because they were made here."""
        self = cls.__new__(cls)
        self.q, self.scale, self.K, self.format, self.wide = q, scale, K, format, wide
        return self

    def dequantize(self, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The values that the rows stand for, rounded to dtype."""
        q, scale, K = self.q, self.scale, self.K
        M, dev = q.shape[0], q.get_device()
        if out is None:
            dt, ldy = _DT.get(dtype), K
            if dt is None:
                _refuse(hb.ERR_DTYPE, "dequantize: result in %s" % dtype)
            out = q.new_empty((M, K), dtype=dtype)
        else:
            ldy, dt = _matrix(out, "out", K, M, dev), _dtype(out, "out")
            _given(out, "out")
        ldq, lds = (q.stride(0), scale.stride(0)) if M > 1 else (q.shape[1], scale.shape[1])
        _on(dev, _dequantize)(q.data_ptr(), ldq, scale.data_ptr(), lds, M, K, FORMATS[self.format], _bits(self.wide), out.data_ptr(), ldy, dt, _stream(dev))
        return out


def quantize_rows(x: torch.Tensor, format: str = "nvfp4", scale: float = 1.0, routing: Optional[Routing] = None, n_rows: Optional[int] = None) -> Fp4Rows:
    """x in 4 bits. scale: the 32-bit scale of an "nvfp4" matrix; blocks' own scales reach from 2^-9 to 448 times it, so that max|x| / 2688 uses them fully. With a
    routing the rows come in expert order (n_rows: the capacity, default tokens * top_k; rows that no choice fills are left alone). Rows start 16 bytes
    apart or a multiple of it. Blocks whose largest element is below 0.1 scale lose bits of their own scale (of normal rows of deviation 0.02 scale 10 % are rounded off as of larger ones, of 0.01 13 %),
    and below 0.006 scale they become zeros."""
    fmt, wide = _format(format), _wide(scale, format)
    _no_gradient(x, "x", "4-bit rows have")
    ldx, dt, dev = _matrix(x, "x", dev=None if routing is None else routing.dev), _dtype(x, "x"), x.get_device()
    M, K = x.shape
    n = M if routing is None else (routing.tokens * routing.top_k if n_rows is None else n_rows)
    blocks = (K + BLOCK[format] - 1) // BLOCK[format]
    width = (K + 1) // 2
    pitch = _pad16(width)
    q, s = x.new_empty((n, pitch), dtype=torch.uint8), x.new_empty((n, blocks), dtype=torch.uint8)
    _on(dev, _quantize)(x.data_ptr(), ldx, M, K, dt, fmt, _bits(wide), routing.at if routing is not None else 0, q.data_ptr(), pitch, s.data_ptr(), blocks, n, _stream(dev))
    return Fp4Rows._made(q if pitch == width else q[:, :width], s, K, format, wide)


class Fp4Linear:
    """y = x W^T (+ bias) with W in 4-bit floating point: weight uint8 [N, (K + 1) // 2] or [experts, N, (K + 1) // 2], scale (bytes of e4m3 or powers of
    two) [.., N, blocks], tensor_scale fp32 [1] or [experts], by which each matrix is multiplied (default ones), bias fp32 [N] or [experts, N]. The rows of x are quantised to the same
    format within the call, "nvfp4" with the 32-bit scale x_scale, which should suit them as quantize_rows's scale does: the default is for rows of order 1, and rows of order 0.002 become zeros by it. K: the width, where it is odd. Scales, and weights whose rows do not start on 16-byte
    boundaries, are laid out anew once, here. A result's rows beyond the last expert's are left alone. For serving: an input that requires a gradient is refused."""

    def __init__(self, weight: torch.Tensor, scale: torch.Tensor, tensor_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                 format: str = "nvfp4", x_scale: float = 1.0, K: Optional[int] = None):
        self.format, self.fmt = format, _format(format)
        weight, scale = _bytes(weight, "Fp4Linear: weight"), _bytes(scale, "Fp4Linear: scale")
        if weight.dim() not in (2, 3) or not weight.is_cuda:
            _refuse(hb.ERR_INVALID_ARG, "Fp4Linear: weight must be a CUDA tensor [N, K / 2] or [experts, N, K / 2]")
        self.experts = weight.shape[0] if weight.dim() == 3 else 0
        self.N, width = weight.shape[-2:]
        self.K = 2 * width if K is None else K
        if (self.K + 1) // 2 != width:
            _refuse(hb.ERR_COUNT_MISMATCH, "Fp4Linear: rows of %d bytes for K = %d" % (width, self.K))
        self.device, self.dev = weight.device, weight.get_device()
        G = max(self.experts, 1)
        blocks = (self.K + BLOCK[format] - 1) // BLOCK[format]
        if scale.shape != weight.shape[:-1] + (blocks,):
            _refuse(hb.ERR_COUNT_MISMATCH, "Fp4Linear: scale is %s, expected %s" % (tuple(scale.shape), tuple(weight.shape[:-1] + (blocks,))))
        if scale.get_device() != self.dev:
            _refuse(hb.ERR_INVALID_ARG, "Fp4Linear: scale must be on cuda:%d" % self.dev)
        if tensor_scale is None:
            tensor_scale = torch.ones(G, dtype=torch.float32, device=self.device)
        _vector(tensor_scale, "tensor_scale", torch.float32, G, self.dev)
        if bias is not None:
            _vector(bias, "bias", torch.float32, G * self.N, self.dev)
        self.x_scale = _wide(x_scale, format)
        if not weight.is_contiguous() or width % 16 or weight.data_ptr() % 16:
            padded = torch.zeros(weight.shape[:-1] + (_pad16(width),), dtype=torch.uint8, device=self.device)
            padded[..., :width] = weight
            weight = padded
        self.weight, self.tensor_scale, self.bias = weight, tensor_scale, bias
        self.ldw = weight.shape[-1]
        self._rows_scale = scale.contiguous()  # kept for copies
        self.scale = self._laid_out(self.N, self.experts)
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._fixed = (self.fmt, weight.data_ptr(), self.ldw, self.scale.data_ptr(), tensor_scale.data_ptr(), bias.data_ptr() if bias is not None else 0)
        self._status_at = self._status.data_ptr()
        self._x_bits = _bits(self.x_scale)
        self._need = {}  # scratch bytes by number of rows

    def _laid_out(self, N: int, groups: int) -> torch.Tensor:
        """The scales as the tensor cores take them, in groups of N rows."""
        out = torch.empty(max(hb.hccl_fp4_weight_scale_bytes(N, self.K, groups, self.fmt), 16), dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.dev):
            hb.hccl_fp4_weight_scales(self._rows_scale.data_ptr(), self._rows_scale.shape[-1], N, self.K, groups, self.fmt, out.data_ptr(), _stream(self.dev))
        return out

    def __reduce__(self):  # a copy has weights, and their addresses, of its own
        return Fp4Linear, (self.weight[..., : (self.K + 1) // 2], self._rows_scale, self.tensor_scale, self.bias, self.format, self.x_scale, self.K)

    @classmethod
    def from_float(cls, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, format: str = "nvfp4", x_scale: float = 1.0) -> "Fp4Linear":
        """Quantises a weight matrix (or one for each expert), each "nvfp4" matrix with the scale max|w| / 2688. Of a parameter, its values."""
        weight = weight.detach()
        _format(format)
        if weight.dim() not in (2, 3):
            _refuse(hb.ERR_INVALID_ARG, "Fp4Linear: weight must have two or three dimensions, not %d" % weight.dim())
        each = weight if weight.dim() == 3 else weight[None]
        wide = [1.0] * each.shape[0]
        if format == "nvfp4" and weight.numel():
            top = each.abs().amax((1, 2)).float()
            wide = torch.where(torch.isfinite(top), (top / top.new_tensor(2688.0)).clamp(1e-30, 1e30), 1.0).tolist()
        rows = [quantize_rows(w, format, s) for w, s in zip(each, wide)]
        q, s = (torch.stack([getattr(r, n) for r in rows]).view(weight.shape[:-1] + (-1,)) if rows and weight.numel() else
                torch.zeros(weight.shape[:-1] + (width,), dtype=torch.uint8, device=weight.device)
                for n, width in (("q", (weight.shape[-1] + 1) // 2), ("scale", -(-weight.shape[-1] // BLOCK[format]))))
        return cls(q, s, torch.tensor(wide, dtype=torch.float32, device=weight.device) if wide else None, bias, format, x_scale, weight.shape[-1])

    def _out(self, out, M, dtype):
        """The result, its row distance and its type."""
        if out is None:
            if dtype not in _DT:
                _refuse(hb.ERR_DTYPE, "Fp4Linear: result in %s" % dtype)
            return self.weight.new_empty((M, self.N), dtype=dtype), self.N, _DT[dtype]
        ldy, dt = _matrix(out, "out", self.N, M, self.dev), _dtype(out, "out")
        _given(out, "out")
        return out, ldy, dt

    def _which(self, routing, offsets):
        if self.experts and (routing is None) == (offsets is None):
            _refuse(hb.ERR_INVALID_ARG, "Fp4Linear over experts takes a routing or offsets")
        if not self.experts and (routing is not None or offsets is not None):
            _refuse(hb.ERR_INVALID_ARG, "Fp4Linear with one matrix takes neither a routing nor offsets")
        if routing is not None and (routing.experts != self.experts or routing.dev != self.dev):
            _refuse(hb.ERR_COUNT_MISMATCH, "Fp4Linear: routing over %d experts on %s" % (routing.experts, routing.device))

    def _args(self, M, dt, x_bits, y, ldy, offsets, stream):
        """The call's record, and the scratch to hold until it is made."""
        if offsets is not None:
            _vector(offsets, "offsets", torch.int32, self.experts + 1, self.dev)
            offsets = offsets.data_ptr()
        need = self._need.get(M)
        if need is None:
            need = self._need[M] = max(hb.hccl_fp4_scratch_bytes(M, self.N, self.K, self.experts, self.fmt), 128)
        hold, at = _scratch.get(self.dev, stream, need)
        fmt, w, ldw, w_scale, w_wide, bias = self._fixed
        return (M, self.N, self.K, self.experts, dt, fmt, x_bits, w, ldw, w_scale, w_wide, bias, offsets or 0, y, ldy, at, need, self._status_at), hold

    def __call__(self, x: torch.Tensor, routing: Optional[Routing] = None, offsets: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [M, K]. Over experts: with a routing, x holds tokens and row r of the result belongs to choice source[r]; with offsets (int32
        [experts + 1], on the device) x is in expert order already."""
        dev = self.dev
        _no_gradient(x, "x", "4-bit rows have")
        ldx, dt = _matrix(x, "x", self.K, None, dev), _dtype(x, "x")
        self._which(routing, offsets)
        M, record = x.shape[0], 0
        if routing is not None:
            if M != routing.tokens:
                _refuse(hb.ERR_COUNT_MISMATCH, "Fp4Linear: %d tokens, the routing has %d" % (M, routing.tokens))
            M, record, offsets = M * routing.top_k, routing.at, routing.offsets
        y, ldy, y_dt = self._out(out, M, x.dtype)
        stream = _stream(dev)
        args, hold = self._args(M, y_dt, self._x_bits, y.data_ptr(), ldy, offsets, stream)
        _on(dev, _linear)(*args, x.data_ptr(), ldx, dt, record, stream)
        return y

    def matmul(self, rows: Fp4Rows, offsets: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """The product alone, of rows that are in 4 bits already (quantize_rows; received from an exchange)."""
        if rows.format != self.format:
            _refuse(hb.ERR_DTYPE, "Fp4Linear: rows in %s, weights in %s" % (rows.format, self.format))
        if rows.K != self.K:
            _refuse(hb.ERR_COUNT_MISMATCH, "Fp4Linear: rows of %d elements, expected %d" % (rows.K, self.K))
        ldq, lds = _matrix(rows.q, "q", dev=self.dev), _matrix(rows.scale, "scale", dev=self.dev)
        self._which(None, offsets)
        M = rows.q.shape[0]
        y, ldy, y_dt = self._out(out, M, dtype)
        stream = _stream(self.dev)
        args, hold = self._args(M, y_dt, _bits(rows.wide), y.data_ptr(), ldy, offsets, stream)
        _on(self.dev, _matmul)(*args, rows.q.data_ptr(), ldq if M > 1 else _pad16(ldq), rows.scale.data_ptr(), lds, stream)
        return y

    def check(self):
        """Synchronises and raises if a product failed on the device since the last check (its result is then undefined)."""
        torch.cuda.synchronize(self.device)
        st = int(self._status.item())
        if st != hb.OK:
            self._status.zero_()
            raise hb.HcclError(st, "Fp4Linear")


class FewTokens:
    """A whole expert layer for a few tokens (at most 64) in two kernels: y[t] = sum over k of weights[t, k] down_e(h_e), e = ids[t, k]. gated: up is [experts, 2 I, H] with the
    gate's rows first, h = act(gate) * other; otherwise up is [experts, I, H] and h = act(up(x)). down is [experts, H, I], of the same format. The weights
    are in 4 bits, activations keep 22 bits below the largest of up to 1024 neighbours: where up and down quantise the rows that they are called with to 4 bits, this does not, so that it is nearer to the
    layer in floating point than down(act(up(x))). For serving: an input that requires a gradient is refused.

    When it is faster than the four calls (up with the routing, activate, down, combine). Called from Python, where those cost the host 44 us: up to about 8 tokens, small layers up to 16. In a captured
    graph: where the experts' weights are the time (2 of 8 of 4096 x 4096, 8 of 64 of 2048 x 1024 and larger) the two take about the same for one to eight tokens (0.9 to 1.15 times their time); small layers and
    more tokens are slower (one token through 2 of 8 experts of 512 x 512 21 us against 17; 16 tokens 1.1 to 2.3 times, 64 tokens 1.5 to 5.6 times)."""

    def __init__(self, up: Fp4Linear, down: Fp4Linear, act: str = "silu", gated: bool = True):
        if act not in ACTS:
            _refuse(hb.ERR_INVALID_ARG, "FewTokens: act %r, expected one of %s" % (act, ", ".join(ACTS)))
        if not up.experts or up.experts != down.experts or up.dev != down.dev:
            _refuse(hb.ERR_INVALID_ARG, "FewTokens: up and down must be over the same number of experts, on one device")
        if up.format != down.format:
            _refuse(hb.ERR_DTYPE, "FewTokens: up in %s, down in %s" % (up.format, down.format))
        if up.N != (2 if gated else 1) * down.K or down.N != up.K:
            _refuse(hb.ERR_COUNT_MISMATCH, "FewTokens: layers are %d -> %d and %d -> %d" % (up.K, up.N, down.K, down.N))
        self.up, self.down, self.act, self.gated = up, down, act, bool(gated)
        self.H, self.dev, self.device = up.K, up.dev, up.device
        _, w_up, ld_up, s_up, g_up, b_up = up._fixed
        _, w_down, ld_down, s_down, g_down, b_down = down._fixed
        if gated and down.K % 128:  # the halves' scales begin on tiles of their own
            self._up_scale = up._laid_out(down.K, 2 * up.experts)
            s_up = self._up_scale.data_ptr()
        self.record = hb.ExpertsFp4(up.K, down.K, up.experts, up.fmt, ACTS[act], 1 if gated else 0, w_up, ld_up, s_up, g_up, b_up, w_down, ld_down, s_down, g_down, b_down)
        hb.hccl_expert_layer_scratch_bytes(self.record, 1, 1)  # refuses sizes that the kernels do not take
        self._at = C.addressof(self.record)
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._status_at = self._status.data_ptr()
        self._need = {}  # scratch bytes by tokens and top_k

    def __reduce__(self):  # the record holds addresses
        return FewTokens, (self.up, self.down, self.act, self.gated)

    def __call__(self, x: torch.Tensor, routing: Routing, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [tokens, H], its routing; returns [tokens, H] in x's type."""
        dev, T, k = self.dev, routing.tokens, routing.top_k
        _no_gradient(x, "x", "FewTokens has")
        _no_gradient(routing.weights, "the routing's weights", "FewTokens has")
        ldx, dt = _matrix(x, "x", self.H, T, dev), _dtype(x, "x")
        if routing.experts != self.up.experts or routing.dev != dev:
            _refuse(hb.ERR_COUNT_MISMATCH, "FewTokens: routing over %d experts on %s" % (routing.experts, routing.device))
        need = self._need.get((T, k))
        if need is None:
            if T > hb.MAX_FEW_TOKENS:
                _refuse(hb.ERR_INVALID_ARG, "FewTokens: %d tokens, at most %d" % (T, hb.MAX_FEW_TOKENS))
            need = self._need[T, k] = hb.hccl_expert_layer_scratch_bytes(self.record, T, k)
        out, ldy = _new(out, T, self.H, x, "out", dev)
        stream = _stream(dev)
        hold, at = _scratch.get(dev, stream, need)
        _on(dev, _layer)(self._at, x.data_ptr(), ldx, dt, routing.at, out.data_ptr(), ldy, at, need, self._status_at, stream)
        return out

    def check(self):
        """Synchronises and raises if a call failed on the device since the last check (its result is then undefined)."""
        torch.cuda.synchronize(self.device)
        st = int(self._status.item())
        if st != hb.OK:
            self._status.zero_()
            raise hb.HcclError(st, "FewTokens")
