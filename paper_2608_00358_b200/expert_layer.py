"""An expert layer over R virtual ranks, one expert to a rank: the operators of experts.py around the device-resident AllToAllv.

Every rank routes its own tokens; its row of the R x R count matrix is what ``hccl_route`` wrote. Rows travel in 8 bits, each with its
scale, straight from ``hccl_quantize_rows_i8`` to the rank of their expert; there they are multiplied; the results travel back by the
transposed counts and are summed with the routing weights. Nothing of it waits for the host: counts, displacements and
offsets stay on the device (the device-resident exchange of Sec. IV-B.2), so a whole forward pass can be captured in a CUDA graph.

    python -m paper_2608_00358_b200.expert_layer --ranks 8 --tokens 512 --hidden 1024 --inner 2048 --top-k 2
"""
from __future__ import annotations

import argparse
from typing import List

import torch

from . import binding as hb
from .experts import Int8Linear, Router, Routing, _dtype, _matrix, _no_gradient, _pad16, _quantize, _refuse, combine
from .runtime import DeviceCollective


def check_experts(router: Router, up: List[Int8Linear], down: List[Int8Linear], dev: int):
    """Refuses experts that do not fit the router or each other: one up and one down for each rank, each over one expert on device number `dev`."""
    if len(up) != router.experts or len(down) != router.experts:
        _refuse(hb.ERR_COUNT_MISMATCH, "ExpertParallel: %d and %d experts for %d ranks" % (len(up), len(down), router.experts))
    for r, (u, d) in enumerate(zip(up, down)):
        if u.experts != 1 or d.experts != 1 or u.dev != dev or d.dev != dev:
            _refuse(hb.ERR_INVALID_ARG, "ExpertParallel: rank %d's layers must be over one expert each, on cuda:%d" % (r, dev))
        if u.K != up[0].K or d.K != u.N or d.N != u.K:
            _refuse(hb.ERR_COUNT_MISMATCH, "ExpertParallel: rank %d's layers are %d -> %d and %d -> %d, the first takes %d" % (r, u.K, u.N, d.K, d.N, up[0].K))


class ExpertParallel:
    """Buffers and plans for `tokens` tokens on each of `ranks` ranks. up: Int8Linear [1, inner, hidden] of each rank's expert, down: [1, hidden, inner];
    act: what stands between them."""

    def __init__(self, router: Router, up: List[Int8Linear], down: List[Int8Linear], tokens: int, act=torch.nn.functional.silu, device="cuda"):
        self.dev = torch.empty(0, device=device).get_device()
        check_experts(router, up, down, self.dev)
        R, k, hidden = router.experts, router.top_k, up[0].K
        self.router, self.up, self.down, self.act = router, up, down, act
        self.R, self.tokens, self.hidden = R, tokens, hidden
        self.send_rows, self.recv_rows = tokens * k, tokens * R  # a token chooses an expert at most once
        i32, i64 = dict(dtype=torch.int32, device=device), dict(dtype=torch.int64, device=device)
        self.counts = torch.zeros((R, R), **i64)  # [source, destination]; hccl_route of rank s writes row s
        self.counts_back = torch.zeros((R, R), **i64)
        shape = (tokens, k)
        self.routing = [Routing(torch.empty(shape, **i32), torch.empty(shape, dtype=torch.float32, device=device), self.counts[r], torch.empty(R + 1, **i32),
                                torch.empty(shape, **i32), torch.empty(tokens * k, **i32)) for r in range(R)]
        # a row on the way: hidden bytes, then its scale, up to a multiple of 16 bytes
        self.at = _pad16(hidden)
        self.row = self.at + 16
        byte = dict(dtype=torch.int8, device=device)
        self.send = [torch.zeros((self.send_rows, self.row), **byte) for _ in range(R)]
        self.recv = [torch.zeros((self.recv_rows, self.row), **byte) for _ in range(R)]
        self.scale = torch.zeros(max(self.send_rows, 1), dtype=torch.float32, device=device)
        self.result = [torch.zeros((self.recv_rows, hidden), dtype=torch.bfloat16, device=device) for _ in range(R)]
        self.back = [torch.zeros((self.send_rows, hidden), dtype=torch.bfloat16, device=device) for _ in range(R)]
        self.offsets = torch.zeros((R, 2), **i32)
        self._out = self._exchange(self.counts, [self.send_rows] * R, [self.recv_rows] * R, self.row // 2, self.send, self.recv)
        self._home = self._exchange(self.counts_back, [self.recv_rows] * R, [self.send_rows] * R, hidden, self.result, self.back)

    def _exchange(self, counts, send_rows, recv_rows, row_elems, send, recv):
        plan = hb.hccl_plan_alltoallv_dynamic(self.R, send_rows, recv_rows, hb.BF16, row_elems)
        plan.set_dynamic_metadata(counts.data_ptr())
        dc = DeviceCollective(plan)
        dc.set_buffers([t.data_ptr() for t in send], [t.data_ptr() for t in recv], keep=(send, recv, counts))
        return dc

    def forward(self, x: List[torch.Tensor], logits: List[torch.Tensor]) -> List[torch.Tensor]:
        """x[r] [tokens, hidden] and logits[r] [tokens, ranks] of every rank; returns each rank's [tokens, hidden] in bf16."""
        if len(x) != self.R or len(logits) != self.R:
            _refuse(hb.ERR_COUNT_MISMATCH, "ExpertParallel: inputs of %d and %d ranks, expected %d" % (len(x), len(logits), self.R))
        for t in x:
            _no_gradient(t, "x")
        rows = [(_matrix(t, "x", self.hidden, self.tokens, self.dev), _dtype(t, "x")) for t in x]
        for t in logits:
            _matrix(t, "logits", self.R, self.tokens, self.dev), _dtype(t, "logits")
        stream = torch.cuda.current_stream()
        for r, (ld, dt) in enumerate(rows):
            self.router.route(logits[r], out=self.routing[r])
            _quantize(x[r].data_ptr(), ld, self.tokens, self.hidden, dt, self.routing[r].at, self.send[r].data_ptr(), self.row,
                      self.send_rows, self.scale.data_ptr(), stream.cuda_stream)
            self.send[r][:, self.at: self.at + 4] = self.scale[: self.send_rows].view(torch.int8).view(-1, 4)
        self._out.execute(stream)
        self.counts_back.copy_(self.counts.t())
        self.offsets[:, 1] = self.counts.sum(0)
        for r in range(self.R):
            scale = self.recv[r][:, self.at: self.at + 4].contiguous().view(torch.float32).view(-1)
            h = self.up[r].matmul(self.recv[r][:, : self.hidden], scale, offsets=self.offsets[r], dtype=torch.bfloat16)
            self.down[r](self.act(h), offsets=self.offsets[r], out=self.result[r])
        self._home.execute(stream)
        return [combine(self.back[r], self.routing[r]) for r in range(self.R)]

    def check(self):
        """Synchronises; raises if an exchange or a product failed on the device."""
        self._out.check()
        self._home.check()
        for lin in self.up + self.down:
            lin.check()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--ranks", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=512, help="of each rank")
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=2048)
    ap.add_argument("--top-k", type=int, default=2)
    ap.add_argument("--iters", type=int, default=20)
    a = ap.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)
    R = a.ranks

    def matrix(n, k):
        return torch.randn((1, n, k), device="cuda", generator=g) * k ** -0.5

    ups, downs = [matrix(a.inner, a.hidden) for _ in range(R)], [matrix(a.hidden, a.inner) for _ in range(R)]
    layer = ExpertParallel(Router(R, a.top_k), [Int8Linear.from_float(w) for w in ups], [Int8Linear.from_float(w) for w in downs], a.tokens)
    x = [torch.randn((a.tokens, a.hidden), device="cuda", generator=g).bfloat16() for _ in range(R)]
    logits = [torch.randn((a.tokens, R), device="cuda", generator=g) for _ in range(R)]
    y = layer.forward(x, logits)
    layer.check()
    # the same layer in 32-bit floating point, on one rank's tokens
    w, ids = torch.softmax(logits[0], -1).topk(a.top_k)
    w = w / w.sum(-1, keepdim=True)
    want = torch.zeros((a.tokens, a.hidden), device="cuda")
    for e in range(R):
        h = torch.nn.functional.silu(x[0].float() @ ups[e][0].t()) @ downs[e][0].t()
        want += torch.where(ids == e, w, 0.0).sum(-1, keepdim=True) * h
    err = float((y[0].float() - want).norm() / want.norm())
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.iters):
        layer.forward(x, logits)
    end.record()
    torch.cuda.synchronize()
    print("%d ranks x %d tokens, %d -> %d -> %d, top %d: %.1f us a pass; against 32-bit floating point: %.2f %% (8-bit weights and rows)"
          % (R, a.tokens, a.hidden, a.inner, a.hidden, a.top_k, start.elapsed_time(end) * 1e3 / a.iters, 100 * err))


if __name__ == "__main__":
    main()
