"""Expert layers on torch tensors: routing, dispatch and combine of rows, linear layers in 8-bit integers.

The operators are the C calls of include/hccl.h (``hccl_route`` and the ones after it); this module checks tensors,
supplies outputs and workspaces, and joins the gradients to torch's autograd. Everything runs on the current stream of
the tensors' device; nothing here computes, and there is no CPU form. Host threads may share a router or a layer.

    router = Router(experts=64, top_k=8, score="sigmoid", renormalise=True)
    r = router.route(logits, bias=balance)            # who goes where, with which weight
    y = up(x, routing=r)                              # Int8Linear over experts: rows gathered, quantised, multiplied
    out = combine(down(act(y), offsets=r.offsets), r) # back to tokens

With real exchanges between ranks, ``dispatch`` (or ``quantize_rows(x, routing=r)`` for half the bytes) lays out the send
buffer of an AllToAllv, and ``r.counts`` is the rank's row of its count matrix when each rank holds one expert.
"""
from __future__ import annotations

import ctypes as C
import threading
from typing import Optional

import torch
from torch.autograd import forward_ad as _forward_ad
from torch.autograd.function import once_differentiable

from . import binding as hb

_route, _route_backward = hb.packed("hccl_route"), hb.packed("hccl_route_backward")
_c_dispatch, _c_dispatch_backward = hb.packed("hccl_dispatch"), hb.packed("hccl_dispatch_backward")
_c_combine, _c_combine_backward = hb.packed("hccl_combine"), hb.packed("hccl_combine_backward")
_quantize, _matmul, _linear = hb.packed("hccl_quantize_rows_i8"), hb.packed("hccl_matmul_i8"), hb.packed("hccl_linear_i8")
_DT = {torch.float32: hb.FP32, torch.bfloat16: hb.BF16, torch.float16: hb.FP16}
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_capturing = torch._C._cuda_isCurrentStreamCapturing if hasattr(torch._C, "_cuda_isCurrentStreamCapturing") else torch.cuda.is_current_stream_capturing
_written = torch._C._increment_version if hasattr(torch._C, "_increment_version") else torch.autograd.graph.increment_version  # of a tuple of tensors
_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _refuse(status: int, what: str):
    raise hb.HcclError(status, what)


def _no_tangent(t: torch.Tensor, what: str):
    """Refuses a dual number of forward-mode differentiation: the kernels would see its value alone and its tangent would be lost."""
    if _forward_ad.unpack_dual(t).tangent is not None:
        _refuse(hb.ERR_INVALID_ARG, "%s has a tangent; there is no forward-mode derivative" % what)


def _no_gradient(t: torch.Tensor, what: str, of: str = "8-bit rows have"):
    """Refuses what autograd would follow: rows in 8 or 4 bits have no gradient, and a result that only looks differentiable stops training without a word."""
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(hb.ERR_INVALID_ARG, "%s requires a gradient, and %s none: detach it or call under torch.no_grad()" % (what, of))


def _given(t: torch.Tensor, what: str):
    """A caller's output is about to be written: autograd, which may hold it for a gradient, is to know as it does of torch's own writes."""
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(hb.ERR_INVALID_ARG, "%s: an output that requires a gradient" % what)
    _written((t,))


def _matrix(t: torch.Tensor, what: str, cols: Optional[int] = None, rows: Optional[int] = None, dev: Optional[int] = None) -> int:
    """Checks a 2-d matrix with adjacent columns on CUDA device number `dev` (None: any); returns the distance between its rows."""
    try:
        n, m = t.shape
    except ValueError:
        _refuse(hb.ERR_INVALID_ARG, "%s must have two dimensions, not %d" % (what, t.dim()))
    at = t.get_device()
    if at < 0 or (dev is not None and at != dev):
        _refuse(hb.ERR_INVALID_ARG, "%s must be on %s, not %s" % (what, "a CUDA device" if dev is None else "cuda:%d" % dev, t.device))
    if (cols is not None and m != cols) or (rows is not None and n != rows):
        _refuse(hb.ERR_COUNT_MISMATCH, "%s is [%d, %d], expected [%s, %s]" % (what, n, m, "any" if rows is None else rows, "any" if cols is None else cols))
    if _forward_ad._current_level >= 0:
        _no_tangent(t, what)
    ld, step = t.stride()
    if step != 1 and m > 1 and n:
        _refuse(hb.ERR_ALIGNMENT, "%s must have adjacent columns" % what)
    return ld if n > 1 else max(ld, m)


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DT.get(t.dtype)
    if d is None:
        _refuse(hb.ERR_DTYPE, "%s is %s" % (what, t.dtype))
    return d


def _vector(t: torch.Tensor, what: str, dtype: torch.dtype, numel: int, dev: int):
    if t.dtype != dtype:
        _refuse(hb.ERR_DTYPE, "%s is %s, expected %s" % (what, t.dtype, dtype))
    if t.numel() != numel:
        _refuse(hb.ERR_COUNT_MISMATCH, "%s has %d elements, expected %d" % (what, t.numel(), numel))
    if t.get_device() != dev or not t.is_contiguous():
        _refuse(hb.ERR_INVALID_ARG, "%s must be contiguous and on cuda:%d" % (what, dev))
    if _forward_ad._current_level >= 0:
        _no_tangent(t, what)


def _same_type(a: torch.Tensor, b: torch.Tensor, what: str):
    if a.dtype != b.dtype:
        _refuse(hb.ERR_DTYPE, "%s: %s and %s" % (what, a.dtype, b.dtype))


def _on(dev: int, call):
    """The call with device number `dev` current; its last argument is that device's stream."""
    if dev == _current_device():
        return call

    def there(*args):
        with torch.cuda.device(dev):
            call(*args)
    return there


class _Scratch(threading.local):
    """Device memory for the calls' own use, one piece for each host thread and stream. What a call leaves there, the next call on that stream may write over, whichever object makes it. Calls on different
    streams do not share a piece, nor do threads on one stream: a call makes up to two launches, and another thread's may come between them. A call that is captured
    into a CUDA graph gets memory of the graph's own, since the graph may be replayed on any stream, beside later calls."""

    def __init__(self):
        self._of = {}

    def get(self, dev: int, stream: int, nbytes: int):
        """(tensor, address) of at least nbytes on device number `dev` for a call on its current stream `stream`; hold the tensor until the call is made."""
        if _capturing():
            t = torch.empty(nbytes, dtype=torch.uint8, device="cuda:%d" % dev)
            return t, t.data_ptr()
        key = (dev, stream)
        have = self._of.get(key)
        if have is None or have[2] < nbytes:
            t = torch.empty(nbytes, dtype=torch.uint8, device="cuda:%d" % dev)
            have = self._of[key] = (t, t.data_ptr(), nbytes)
        return have[:2]


_scratch = _Scratch()


class Routing:
    """Which token goes to which expert (hccl_routing_t), as tensors: ids, weights, slots [tokens, top_k]; counts [experts];
    offsets [experts + 1]; source [tokens * top_k]. Rows of expert e, in expert order, are offsets[e]:offsets[e + 1]."""

    __slots__ = ("ids", "weights", "counts", "offsets", "slots", "source", "tokens", "top_k", "experts", "device", "dev", "record", "at")

    def __init__(self, ids, weights, counts, offsets, slots, source):
        if ids.dim() != 2 or not ids.is_cuda:
            _refuse(hb.ERR_INVALID_ARG, "Routing: ids must be a CUDA tensor [tokens, top_k]")
        self.tokens, self.top_k = ids.shape
        self.experts, self.device, self.dev = counts.numel(), ids.device, ids.get_device()
        n = self.tokens * self.top_k
        for t, what, dt, numel in ((ids, "ids", torch.int32, n), (weights, "weights", torch.float32, n), (counts, "counts", torch.int64, self.experts),
                                   (offsets, "offsets", torch.int32, self.experts + 1), (slots, "slots", torch.int32, n),
                                   (source, "source", torch.int32, n)):
            _vector(t, what, dt, numel, self.dev)
        self.ids, self.weights, self.counts, self.offsets, self.slots, self.source = ids, weights, counts, offsets, slots, source
        self.record = hb.RoutingRecord(self.tokens, self.top_k, self.experts, ids.data_ptr(), weights.data_ptr(), counts.data_ptr(),
                                       offsets.data_ptr(), slots.data_ptr(), source.data_ptr())
        self.at = C.addressof(self.record)

    def __reduce__(self):  # copies and pickles are made from the tensors: the record holds addresses
        return Routing, (self.ids, self.weights, self.counts, self.offsets, self.slots, self.source)


class Router:
    """How tokens choose experts (hccl_router_t). score "softmax" or "sigmoid"; groups > 1: only the experts of the top_groups best
    groups are eligible, a group's score being the sum of its group_best (1 or 2) largest keys."""

    def __init__(self, experts: int, top_k: int, score: str = "softmax", groups: int = 1, top_groups: int = 1, group_best: int = 1,
                 renormalise: bool = True, scale: float = 1.0):
        if score not in ("softmax", "sigmoid"):
            _refuse(hb.ERR_INVALID_ARG, "Router: score %r" % (score,))
        self.config = hb.RouterConfig(experts, top_k, hb.SCORE_SIGMOID if score == "sigmoid" else hb.SCORE_SOFTMAX, groups, top_groups, group_best,
                                      1 if renormalise else 0, scale)
        hb.hccl_route_workspace_bytes(self.config, 0)  # refuses a configuration that does not hold together
        self.experts, self.top_k = experts, top_k
        self._made_of = (experts, top_k, score, groups, top_groups, group_best, renormalise, scale)
        self._at = C.addressof(self.config)
        self._need = {}  # workspace bytes by number of tokens
        self._untouched = {}  # by device, what calls get that have no use for a workspace

    def __reduce__(self):  # a copy has a configuration, and its address, of its own
        return Router, self._made_of

    def _some(self, dev: int):
        t = torch.empty(hb.ROUTE_NO_WORKSPACE, dtype=torch.uint8, device="cuda:%d" % dev)
        have = self._untouched[dev] = (t, t.data_ptr())
        return have

    def outputs(self, tokens: int, device="cuda") -> Routing:
        """Memory for one routing of `tokens` tokens, to be given as out=."""
        n, i32 = (tokens, self.top_k), dict(dtype=torch.int32, device=device)
        return Routing(torch.empty(n, **i32), torch.empty(n, dtype=torch.float32, device=device),
                       torch.empty(self.experts, dtype=torch.int64, device=device), torch.empty(self.experts + 1, **i32),
                       torch.empty(n, **i32), torch.empty(tokens * self.top_k, **i32))

    def _inputs(self, logits, bias, token_mask, tokens, dev):
        ld = _matrix(logits, "logits", self.experts, tokens, dev)
        dt = _dtype(logits, "logits")
        b = m = 0
        if bias is not None:
            _vector(bias, "bias", torch.float32, self.experts, dev)
            b = bias.data_ptr()
        if token_mask is not None:
            if token_mask.dtype == torch.bool:
                token_mask = token_mask.view(torch.uint8)
            _vector(token_mask, "token_mask", torch.uint8, tokens, dev)
            m = token_mask.data_ptr()
        return ld, dt, b, m

    def _run(self, logits, bias, token_mask, out):
        dev, tokens = out.dev, out.tokens
        ld, dt, b, m = self._inputs(logits, bias, token_mask, tokens, dev)
        if out.experts != self.experts or out.top_k != self.top_k:
            _refuse(hb.ERR_COUNT_MISMATCH, "route: out is for %d tokens, %d experts, top %d" % (tokens, out.experts, out.top_k))
        need = self._need.get(tokens)
        if need is None:
            need = self._need[tokens] = hb.hccl_route_workspace_bytes(self.config, tokens)
        stream = _stream(dev)
        if need <= hb.ROUTE_NO_WORKSPACE:
            hold, ws = self._untouched.get(dev) or self._some(dev)
        else:
            hold, ws = _scratch.get(dev, stream, need)
        _on(dev, _route)(self._at, logits.data_ptr(), ld, dt, b, m, out.at, ws, need, stream)

    def route(self, logits: torch.Tensor, bias: Optional[torch.Tensor] = None, token_mask: Optional[torch.Tensor] = None,
              out: Optional[Routing] = None) -> Routing:
        """logits [tokens, experts]; bias fp32 [experts], added to the scores for the choice only; token_mask [tokens], 0 or False for padding.
        With gradients enabled and logits that require them, the result's weights carry the graph."""
        if logits.requires_grad and torch.is_grad_enabled():
            if out is not None:
                _refuse(hb.ERR_INVALID_ARG, "route: out= cannot carry a gradient")
            out = self.outputs(logits.shape[0], logits.device)
            w = _Route.apply(logits, self, bias, token_mask, out)
            return Routing(out.ids, w, out.counts, out.offsets, out.slots, out.source)
        if out is None:
            out = self.outputs(logits.shape[0], logits.device)
            self._run(logits, bias, token_mask, out)
            return out
        if out.weights.requires_grad and torch.is_grad_enabled():
            _refuse(hb.ERR_INVALID_ARG, "route: out= has weights that carry a gradient")
        self._run(logits, bias, token_mask, out)
        _written((out.ids, out.weights, out.counts, out.offsets, out.slots, out.source))
        return out

    def backward(self, logits: torch.Tensor, routing: Routing, dweights: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 token_mask: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Gradient of the logits for a gradient of the weights (fp32 [tokens, top_k])."""
        return self._gradient(logits, routing.at, routing.tokens, routing.top_k, routing.dev, dweights, bias, token_mask, out)

    def _gradient(self, logits, routing_at, tokens, top_k, dev, dweights, bias, token_mask, out):
        ld, dt, b, m = self._inputs(logits, bias, token_mask, tokens, dev)
        _vector(dweights, "dweights", torch.float32, tokens * top_k, dev)
        out, ldd = _new(out, tokens, self.experts, logits, "dlogits", dev)
        _on(dev, _route_backward)(self._at, logits.data_ptr(), ld, dt, b, m, routing_at, dweights.data_ptr(), out.data_ptr(), ldd, _stream(dev))
        return out


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, router, bias, token_mask, out):
        router._run(logits, bias, token_mask, out)
        # Not `out` itself: its weights are this function's result and would hold on to it, a cycle that only the collector frees.
        ctx.save_for_backward(logits, bias, token_mask, out.ids)
        ctx.router = router
        return out.weights

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights):
        logits, bias, token_mask, ids = ctx.saved_tensors
        tokens, top_k = ids.shape
        record = hb.RoutingRecord(tokens, top_k, ctx.router.experts, ids.data_ptr())  # the gradient reads the ids alone
        return ctx.router._gradient(logits, C.addressof(record), tokens, top_k, ids.get_device(), dweights.contiguous(), bias, token_mask, None), None, None, None, None


def _new(out, rows, cols, like, what, dev):
    """The output and the distance between its rows: memory of `like`'s type, or the caller's after a check."""
    if out is None:
        return like.new_empty((rows, cols)), cols
    _same_type(out, like, what)
    ld = _matrix(out, what, cols, rows, dev)
    _given(out, what)
    return out, ld


def _weights(weights, routing) -> int:
    if weights is None:
        return routing.weights.data_ptr()
    _vector(weights, "weights", torch.float32, routing.tokens * routing.top_k, routing.dev)
    return weights.data_ptr()


def _dispatch(x, routing, out, n_rows):
    dev = routing.dev
    ldx, dt = _matrix(x, "x", None, routing.tokens, dev), _dtype(x, "x")
    H = x.shape[1]
    if out is None and n_rows is None:
        n_rows = routing.tokens * routing.top_k
    out, ldr = _new(out, n_rows, H, x, "rows", dev)
    _on(dev, _c_dispatch)(x.data_ptr(), ldx, H, dt, routing.at, out.data_ptr(), ldr, out.shape[0], _stream(dev))
    return out


def dispatch(x: torch.Tensor, routing: Routing, out: Optional[torch.Tensor] = None, n_rows: Optional[int] = None) -> torch.Tensor:
    """Rows in expert order: out[slots[t, k]] = x[t]. n_rows (default tokens * top_k): the capacity; choices beyond it are dropped."""
    if x.requires_grad and torch.is_grad_enabled():
        if out is not None:
            _refuse(hb.ERR_INVALID_ARG, "dispatch: out= cannot carry a gradient")
        return _Dispatch.apply(x, routing, n_rows)
    return _dispatch(x, routing, out, n_rows)


def dispatch_backward(drows: torch.Tensor, routing: Routing, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx[t] = sum over k of drows[slots[t, k]]."""
    dev = routing.dev
    ldr, dt = _matrix(drows, "drows", None, None, dev), _dtype(drows, "drows")
    n, H = drows.shape
    out, ldx = _new(out, routing.tokens, H, drows, "dx", dev)
    _on(dev, _c_dispatch_backward)(drows.data_ptr(), ldr, n, H, dt, routing.at, out.data_ptr(), ldx, _stream(dev))
    return out


def _combine(rows, routing, weights, out):
    dev = routing.dev
    ldr, dt = _matrix(rows, "rows", None, None, dev), _dtype(rows, "rows")
    w = _weights(weights, routing)
    n, H = rows.shape
    out, ldy = _new(out, routing.tokens, H, rows, "y", dev)
    _on(dev, _c_combine)(rows.data_ptr(), ldr, n, H, dt, routing.at, w, out.data_ptr(), ldy, _stream(dev))
    return out


def combine(rows: torch.Tensor, routing: Routing, weights: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y[t] = sum over k of weights[t, k] * rows[slots[t, k]]; weights default to the routing's."""
    if torch.is_grad_enabled() and (rows.requires_grad or (routing.weights if weights is None else weights).requires_grad):
        if out is not None:
            _refuse(hb.ERR_INVALID_ARG, "combine: out= cannot carry a gradient")
        return _Combine.apply(rows, routing.weights if weights is None else weights, routing)
    return _combine(rows, routing, weights, out)


def combine_backward(dy: torch.Tensor, rows: torch.Tensor, routing: Routing, weights: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None):
    """(drows, dweights) for a gradient dy of combine's result."""
    dev = routing.dev
    ldr, dt = _matrix(rows, "rows", None, None, dev), _dtype(rows, "rows")
    n, H = rows.shape
    ldy = _matrix(dy, "dy", H, routing.tokens, dev)
    _same_type(dy, rows, "combine backward")
    w = _weights(weights, routing)
    out, ldd = _new(out, n, H, rows, "drows", dev)
    dw = routing.weights.new_empty((routing.tokens, routing.top_k))
    _on(dev, _c_combine_backward)(dy.data_ptr(), ldy, rows.data_ptr(), ldr, n, H, dt, routing.at, w, out.data_ptr(), ldd, dw.data_ptr(), _stream(dev))
    return out, dw


def _cols(t: torch.Tensor) -> torch.Tensor:
    """Adjacent columns and rows that do not overlap, for a gradient that autograd hands over in any layout (expanded over tokens, say)."""
    n, m = t.shape
    return t if (t.stride(1) == 1 or m <= 1) and (t.stride(0) >= m or n <= 1) else t.contiguous()


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, routing, n_rows):
        ctx.save_for_backward(routing.slots)  # for torch's check alone: a routing that was routed into again has no gradient to give
        ctx.routing = routing
        return _dispatch(x, routing, None, n_rows)

    @staticmethod
    @once_differentiable
    def backward(ctx, drows):
        ctx.saved_tensors
        return dispatch_backward(_cols(drows), ctx.routing), None, None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, weights, routing):
        ctx.save_for_backward(rows, weights, routing.slots, routing.offsets)
        ctx.routing = routing
        return _combine(rows, routing, weights, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        rows, weights, _, _ = ctx.saved_tensors
        drows, dw = combine_backward(_cols(dy), rows, ctx.routing, weights)
        return drows, dw.view_as(weights), None


def _pad16(n: int) -> int:
    return (n + 15) // 16 * 16


def quantize_rows(x: torch.Tensor, routing: Optional[Routing] = None, n_rows: Optional[int] = None):
    """(q, scale): 8-bit rows and a scale for each, x[m] ~ q[m] * scale[m]. With a routing the rows come in expert order (n_rows: the
    capacity, default tokens * top_k; rows that no choice fills are left alone). q's rows start 16 bytes apart or a multiple of it."""
    _no_gradient(x, "x")
    ldx, dt, dev = _matrix(x, "x", dev=None if routing is None else routing.dev), _dtype(x, "x"), x.get_device()
    M, K = x.shape
    n = M if routing is None else (routing.tokens * routing.top_k if n_rows is None else n_rows)
    q = torch.empty((n, _pad16(K)), dtype=torch.int8, device=x.device)
    scale = torch.empty(n, dtype=torch.float32, device=x.device)
    _on(dev, _quantize)(x.data_ptr(), ldx, M, K, dt, routing.at if routing is not None else 0, q.data_ptr(), q.shape[1], n, scale.data_ptr(), _stream(dev))
    return q[:, :K], scale


class Int8Linear:
    """y = x W^T (+ bias) with W in 8-bit integers and a scale for each output channel: weight [N, K], or [experts, N, K]; scale and bias
    (fp32) [N] or [experts, N]. The rows of x are quantised within the call, each with a scale of its own. Weights whose rows do not start
    on 16-byte boundaries are laid out anew once, here. A result's rows beyond the last expert's are left alone. For serving: an input that requires a gradient is refused."""

    def __init__(self, weight: torch.Tensor, scale: torch.Tensor, bias: Optional[torch.Tensor] = None):
        if weight.dtype != torch.int8:
            _refuse(hb.ERR_DTYPE, "Int8Linear: weight is %s" % weight.dtype)
        if weight.dim() not in (2, 3) or not weight.is_cuda:
            _refuse(hb.ERR_INVALID_ARG, "Int8Linear: weight must be a CUDA tensor [N, K] or [experts, N, K]")
        self.experts = weight.shape[0] if weight.dim() == 3 else 0
        self.N, self.K = weight.shape[-2:]
        self.device, self.dev = weight.device, weight.get_device()
        rows = max(self.experts, 1) * self.N
        _vector(scale, "scale", torch.float32, rows, self.dev)
        if bias is not None:
            _vector(bias, "bias", torch.float32, rows, self.dev)
        if not weight.is_contiguous() or self.K % 16 or weight.data_ptr() % 16:
            padded = torch.zeros(weight.shape[:-1] + (_pad16(self.K),), dtype=torch.int8, device=self.device)
            padded[..., : self.K] = weight
            weight = padded
        self.weight, self.scale, self.bias = weight, scale, bias
        self.ldw = weight.shape[-1]
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._fixed = (weight.data_ptr(), self.ldw, scale.data_ptr(), bias.data_ptr() if bias is not None else 0)
        self._status_at = self._status.data_ptr()

    def __reduce__(self):  # a copy has weights, and their addresses, of its own
        return Int8Linear, (self.weight[..., : self.K], self.scale, self.bias)

    @classmethod
    def from_float(cls, weight: torch.Tensor, bias: Optional[torch.Tensor] = None) -> "Int8Linear":
        """Quantises a weight matrix (or one for each expert), a scale for each output channel. Of a parameter, its values."""
        weight = weight.detach()
        q, scale = quantize_rows(weight.reshape(-1, weight.shape[-1]))
        return cls(q.reshape(weight.shape), scale.view(weight.shape[:-1]), bias)

    def _args(self, M, a, lda, a_scale, dt, y, ldy, offsets):
        w, ldw, w_scale, bias = self._fixed
        if offsets is not None:
            _vector(offsets, "offsets", torch.int32, self.experts + 1, self.dev)
            offsets = offsets.data_ptr()
        return M, self.N, self.K, self.experts, dt, a, lda, a_scale, w, ldw, w_scale, bias, offsets or 0, y, ldy, self._status_at

    def _out(self, out, M, dtype):
        """The result, its row distance and its type."""
        if out is None:
            if dtype not in _DT:
                _refuse(hb.ERR_DTYPE, "Int8Linear: result in %s" % dtype)
            return torch.empty((M, self.N), dtype=dtype, device=self.device), self.N, _DT[dtype]
        ldy, dt = _matrix(out, "out", self.N, M, self.dev), _dtype(out, "out")
        _given(out, "out")
        return out, ldy, dt

    def _which(self, routing, offsets):
        if self.experts and (routing is None) == (offsets is None):
            _refuse(hb.ERR_INVALID_ARG, "Int8Linear over experts takes a routing or offsets")
        if not self.experts and (routing is not None or offsets is not None):
            _refuse(hb.ERR_INVALID_ARG, "Int8Linear with one matrix takes neither a routing nor offsets")
        if routing is not None and (routing.experts != self.experts or routing.dev != self.dev):
            _refuse(hb.ERR_COUNT_MISMATCH, "Int8Linear: routing over %d experts on %s" % (routing.experts, routing.device))

    def __call__(self, x: torch.Tensor, routing: Optional[Routing] = None, offsets: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [M, K]. Over experts: with a routing, x holds tokens and row r of the result belongs to choice source[r]; with offsets (int32
        [experts + 1], on the device) x is in expert order already."""
        dev, K = self.dev, self.K
        _no_gradient(x, "x")
        ldx, dt = _matrix(x, "x", K, None, dev), _dtype(x, "x")
        self._which(routing, offsets)
        M, record = x.shape[0], 0
        if routing is not None:
            if M != routing.tokens:
                _refuse(hb.ERR_COUNT_MISMATCH, "Int8Linear: %d tokens, the routing has %d" % (M, routing.tokens))
            M, record, offsets = M * routing.top_k, routing.at, routing.offsets
        y, ldy, y_dt = self._out(out, M, x.dtype)
        lda = _pad16(K)
        room = M * lda
        stream = _stream(dev)
        hold, at = _scratch.get(dev, stream, room + 4 * M)
        _on(dev, _linear)(*self._args(M, at, lda, at + room, y_dt, y.data_ptr(), ldy, offsets), x.data_ptr(), ldx, dt, record, stream)
        return y

    def matmul(self, q: torch.Tensor, q_scale: torch.Tensor, offsets: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """The product alone, of rows that are in 8 bits already (quantize_rows; received from an exchange)."""
        if q.dtype != torch.int8:
            _refuse(hb.ERR_DTYPE, "Int8Linear: q is %s" % q.dtype)
        _no_gradient(q_scale, "q_scale")
        lda = _matrix(q, "q", self.K, None, self.dev)
        M = q.shape[0]
        _vector(q_scale, "q_scale", torch.float32, M, self.dev)
        self._which(None, offsets)
        y, ldy, y_dt = self._out(out, M, dtype)
        _on(self.dev, _matmul)(*self._args(M, q.data_ptr(), lda if M > 1 else _pad16(lda), q_scale.data_ptr(), y_dt, y.data_ptr(), ldy, offsets), _stream(self.dev))
        return y

    def check(self):
        """Synchronises and raises if a product failed on the device since the last check (its result is then undefined)."""
        torch.cuda.synchronize(self.device)
        st = int(self._status.item())
        if st != hb.OK:
            self._status.zero_()
            raise hb.HcclError(st, "Int8Linear")
