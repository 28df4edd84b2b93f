"""Expert layers, host side: what the Python layer does before a launch, checked on the CPU with stand-ins for the device's calls."""
import ctypes as C
import os
import re
import struct
import threading

import pytest
import torch

from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex


@pytest.fixture
def no_device(monkeypatch):
    """Device memory from the host's, nothing captured."""
    real = torch.empty
    monkeypatch.setattr(ex.torch, "empty", lambda *a, **kw: real(*a, **{k: v for k, v in kw.items() if k != "device"}))
    monkeypatch.setattr(ex, "_capturing", lambda: False)


def test_scratch_is_not_shared_by_host_threads(no_device):
    """Calls of two launches may interleave between threads on one stream (the library is called without the interpreter's lock): what one thread's first launch
    left for its second must not be another's to write."""
    scratch = ex._Scratch()
    mine = scratch.get(0, 7, 1000)
    seen = []
    t = threading.Thread(target=lambda: seen.append(scratch.get(0, 7, 1000)))
    t.start()
    t.join()
    assert seen[0][1] != mine[1]
    assert scratch.get(0, 7, 500)[1] == mine[1]  # the same thread and stream: the same memory
    assert scratch.get(0, 7, 2000)[0].numel() >= 2000


class Seen(Exception):
    """A launch was reached."""


def layer_without_a_device(monkeypatch, R=2, tokens=3, hidden=32):
    """An ExpertParallel whose first launches only say that they were reached."""
    from paper_2608_00358_b200 import expert_layer as el

    def reached(*a, **kw):
        raise Seen

    class Stream:
        cuda_stream = 0

    layer = object.__new__(el.ExpertParallel)
    layer.R, layer.tokens, layer.hidden, layer.dev = R, tokens, hidden, 0
    layer.router = type("R", (), dict(route=staticmethod(lambda *a, **kw: None), experts=R, top_k=1))()
    layer.routing = [type("P", (), dict(at=0))() for _ in range(R)]
    layer.send = [torch.zeros(tokens, 48, dtype=torch.int8) for _ in range(R)]
    layer.scale, layer.row, layer.at, layer.send_rows = torch.zeros(tokens), 48, 32, tokens
    monkeypatch.setattr(el, "_quantize", reached)
    monkeypatch.setattr(el.torch.cuda, "current_stream", lambda *a: Stream())
    return layer


def on_device(t):
    """A stand-in that says it is on device 0; its address is the host's, which nothing may follow."""
    class There(torch.Tensor):
        def get_device(self):
            return 0

    return t.as_subclass(There)


@pytest.mark.parametrize("what,want", [("few rows", hb.ERR_COUNT_MISMATCH), ("many rows", hb.ERR_COUNT_MISMATCH), ("few columns", hb.ERR_COUNT_MISMATCH), ("columns apart", hb.ERR_ALIGNMENT),
                                       ("host", hb.ERR_INVALID_ARG), ("type", hb.ERR_DTYPE), ("vector", hb.ERR_INVALID_ARG), ("ranks", hb.ERR_COUNT_MISMATCH),
                                       ("logits", hb.ERR_COUNT_MISMATCH), ("nothing", None)])
def test_an_expert_layer_checks_its_inputs_before_the_first_launch(monkeypatch, what, want):
    layer = layer_without_a_device(monkeypatch)
    good = lambda: on_device(torch.zeros(3, 32))  # noqa: E731
    x = [good(), good()]
    x[1] = {"few rows": on_device(torch.zeros(2, 32)), "many rows": on_device(torch.zeros(4, 32)), "few columns": on_device(torch.zeros(3, 31)),
            "columns apart": on_device(torch.zeros(32, 3).t()), "host": torch.zeros(3, 32), "type": on_device(torch.zeros(3, 32).double()),
            "vector": on_device(torch.zeros(96))}.get(what, x[1])
    logits = [on_device(torch.zeros(3, 2)), on_device(torch.zeros(2 if what == "logits" else 3, 2))]
    if what == "ranks":
        x.pop()
    if want is None:
        with pytest.raises(Seen):
            layer.forward(x, logits)
        return
    with pytest.raises(hb.HcclError) as e:
        layer.forward(x, logits)
    assert e.value.status == want


def test_an_expert_layer_checks_its_experts():
    from paper_2608_00358_b200 import expert_layer as el

    def lin(n, k, experts=1, dev=0):
        return type("L", (), dict(N=n, K=k, experts=experts, dev=dev))()

    router = type("R", (), dict(experts=2, top_k=1))()
    up, down = [lin(64, 32), lin(48, 32)], [lin(32, 64), lin(32, 48)]
    for u, d in ((up[:1], down), (up, down[:1]), ([up[0], lin(48, 31)], down), (up, [down[0], lin(32, 64)]), (up, [down[0], lin(31, 48)]),
                 ([lin(64, 32, experts=2), up[1]], down), ([lin(64, 32, experts=0), up[1]], down), (up, [down[0], lin(32, 48, dev=1)])):
        with pytest.raises(hb.HcclError) as e:
            el.check_experts(router, u, d, 0)
        assert e.value.status in (hb.ERR_COUNT_MISMATCH, hb.ERR_INVALID_ARG)
    el.check_experts(router, up, down, 0)


@pytest.mark.parametrize("T,H", [(5, 4), (5, 1), (1, 4), (1, 1), (0, 4), (4, 0)])
def test_a_gradient_of_any_layout_gets_rows_that_the_calls_take(T, H):
    """What autograd hands over is expanded over rows, over columns, over both, or transposed; the C calls want adjacent columns and rows that do not overlap."""
    base = torch.arange(T * H, dtype=torch.float32).view(T, H)
    row, col = torch.arange(H, dtype=torch.float32), torch.arange(T, dtype=torch.float32)[:, None]
    for g in (base, row.expand(T, H), col.expand(T, H), torch.tensor(3.0).expand(T, H), base.t().contiguous().t(), torch.zeros(T, H + 3)[:, :H],
              torch.arange(T + H + 1, dtype=torch.float32).as_strided((T, H), (1, 1))):
        v = ex._cols(g)
        assert torch.equal(v, g)
        assert v.stride(1) == 1 or H <= 1 or T == 0
        assert v.stride(0) >= H or T <= 1
        assert ex._matrix(on_device(v), "g", H, T, 0) >= H  # (of an empty one the strides do not matter)
    wide = torch.zeros(T, H + 3)[:, :H]
    assert ex._cols(wide) is wide  # no copy where none is needed


# ------------------------------------------------------------------------------------------------ the binding's calls with packed arguments
A = 1 << 20  # an aligned address that nothing reads


def packed_calls():
    """What the records must outlive, and for each call its name, arguments that hold together, and (place, value, status) for every place with a refusal of its own. Only
    lists with such a change are handed over: none reaches a device."""
    router = hb.RouterConfig(8, 2, 0, 1, 1, 1, 1, 1.0)
    routing = hb.RoutingRecord(4, 2, 8, A, A, A, A, A, A)
    other = hb.RoutingRecord(5, 2, 8, A, A, A, A, A, A)
    without = hb.RoutingRecord(4, 2, 8, A, A, A, 0, A, A)
    R, P, O, N = C.addressof(router), C.addressof(routing), C.addressof(other), C.addressof(without)
    keep = (router, routing, other, without)
    bad, ali, dty, mism, wsp = hb.ERR_INVALID_ARG, hb.ERR_ALIGNMENT, hb.ERR_DTYPE, hb.ERR_COUNT_MISMATCH, hb.ERR_WORKSPACE
    mm = [4, 8, 32, 0, hb.BF16, A, 32, A, A, 32, A, 0, 0, A, 8, 0]  # M N K groups dtype a lda a_scale w ldw w_scale bias offsets y ldy dev_status
    mm_bad = [(0, -1, bad), (1, -1, bad), (2, hb.MAX_I8_K + 1, bad), (3, 2, bad), (4, 9, dty), (5, 0, bad), (5, A + 8, ali), (6, 16, bad), (6, 40, ali), (7, 0, bad), (7, A + 2, ali),
              (8, 0, bad), (8, A + 1, ali), (9, 16, bad), (9, 40, ali), (10, 0, bad), (10, A + 2, ali), (11, A + 2, ali), (12, A + 2, ali), (13, 0, bad), (13, A + 1, ali), (14, 7, bad), (15, A + 1, ali)]
    return keep, [
        ("hccl_route", [R, A, 8, hb.BF16, 0, 0, P, A, 1 << 20, 0],
         [(0, 0, bad), (1, 0, bad), (1, A + 1, ali), (2, 7, bad), (3, 9, dty), (4, A + 2, ali), (6, 0, bad), (7, 0, bad), (7, A + 4, ali), (8, 0, wsp)]),
        ("hccl_route_backward", [R, A, 8, hb.FP32, 0, 0, P, A, A, 8, 0],
         [(0, 0, bad), (1, 0, bad), (2, 7, bad), (3, 9, dty), (4, A + 2, ali), (6, 0, bad), (7, 0, bad), (7, A + 2, ali), (8, 0, bad), (8, A + 2, ali), (9, 3, bad)]),
        ("hccl_dispatch", [A, 16, 16, hb.BF16, P, A, 16, 8, 0],
         [(0, 0, bad), (0, A + 1, ali), (1, 15, bad), (2, -1, bad), (3, 9, dty), (4, 0, bad), (5, 0, bad), (5, A + 1, ali), (6, 15, bad), (7, -1, bad)]),
        ("hccl_dispatch_backward", [A, 16, 8, 16, hb.BF16, P, A, 16, 0],
         [(0, 0, bad), (0, A + 1, ali), (1, 15, bad), (2, -1, bad), (3, -1, bad), (4, 9, dty), (5, 0, bad), (6, 0, bad), (6, A + 1, ali), (7, 15, bad)]),
        ("hccl_combine", [A, 16, 8, 16, hb.BF16, P, A, A, 16, 0],
         [(0, 0, bad), (0, A + 1, ali), (1, 15, bad), (2, -1, bad), (3, -1, bad), (4, 9, dty), (5, 0, bad), (6, 0, bad), (6, A + 2, ali), (7, 0, bad), (7, A + 1, ali), (8, 15, bad)]),
        ("hccl_combine_backward", [A, 16, A, 16, 8, 16, hb.BF16, P, A, A, 16, A, 0],
         [(0, 0, bad), (1, 15, bad), (2, 0, bad), (2, A + 1, ali), (3, 15, bad), (4, -1, bad), (5, -1, bad), (6, 9, dty), (7, 0, bad), (8, 0, bad), (8, A + 2, ali), (9, 0, bad), (9, A + 1, ali),
          (10, 15, bad), (11, 0, bad), (11, A + 2, ali)]),
        ("hccl_quantize_rows_i8", [A, 32, 4, 32, hb.BF16, P, A, 32, 8, A, 0],
         [(0, 0, bad), (0, A + 1, ali), (1, 31, bad), (2, 5, mism), (3, hb.MAX_I8_K + 1, bad), (4, 9, dty), (5, O, mism), (6, 0, bad), (7, 31, bad), (8, -1, bad), (9, 0, bad), (9, A + 1, ali)]),
        ("hccl_matmul_i8", mm + [0], mm_bad),
        ("hccl_linear_i8", mm + [A, 32, hb.BF16, 0, 0], mm_bad + [(16, 0, bad), (16, A + 1, ali), (17, 31, bad), (18, 9, dty), (19, N, bad)]),
    ]


def plain(name, args):
    """The same through the call itself."""
    if name in ("hccl_matmul_i8", "hccl_linear_i8"):
        m = hb.MatmulI8(*args[:16])
        rest = list(args[16:])
        if name == "hccl_linear_i8":
            rest[3] = C.cast(rest[3], C.POINTER(hb.RoutingRecord)) if rest[3] else None
        return getattr(hb, name)(C.byref(m), *rest)
    typed = {"hccl_route": {0: hb.RouterConfig, 6: hb.RoutingRecord}, "hccl_route_backward": {0: hb.RouterConfig, 6: hb.RoutingRecord}, "hccl_dispatch": {4: hb.RoutingRecord},
             "hccl_dispatch_backward": {5: hb.RoutingRecord}, "hccl_combine": {5: hb.RoutingRecord}, "hccl_combine_backward": {7: hb.RoutingRecord}, "hccl_quantize_rows_i8": {5: hb.RoutingRecord}}[name]
    return getattr(hb, name)(*[(C.cast(a, C.POINTER(typed[i])) if a else None) if i in typed else a for i, a in enumerate(args)])


@pytest.mark.parametrize("at", range(9))
def test_packed_arguments_reach_the_places_of_the_call(at):
    """Every place that the call can refuse, one at a time: the packed call gives the call's own answer."""
    keep, calls = packed_calls()
    name, good, changes = calls[at]
    assert len(good) == hb.CALLS[name] >> 8
    for place, value, want in changes:
        args = list(good)
        args[place] = value
        for call in (lambda: plain(name, args), lambda: hb.packed(name)(*args)):
            with pytest.raises(hb.HcclError) as e:
                call()
            assert e.value.status == want, (name, place, value)


def test_packed_calls_are_those_of_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hccl.h")).read()
    declared = {"hccl_" + n.lower(): int(v, 16) for n, v in re.findall(r"HCCL_CALL_(\w+) = (0x[0-9a-f]+)", text)}
    assert declared == hb.CALLS
    for call in (0, 10, 0x0a01, 0x0b00, 0x1509, -1):
        assert hb._lib.hccl_call_packed(call, b"\0" * 256) == hb.ERR_INVALID_ARG
    assert hb._lib.hccl_call_packed(hb.CALLS["hccl_route"], None) == hb.ERR_INVALID_ARG
    with pytest.raises(struct.error):
        hb.packed("hccl_route")(0, 0)  # too few arguments


@pytest.mark.parametrize("kw", [dict(M=(1 << 31) - 1), dict(M=(1 << 31) - 200), dict(N=(1 << 31) - 1, ldy=1 << 31), dict(N=(1 << 31) - 100, ldy=1 << 31),
                                dict(groups=2, offsets=A, N=(1 << 30) - 1, ldy=1 << 30)])
def test_products_whose_last_tile_would_pass_32_bits_are_refused(kw):
    """A tile's rows and channels are counted in 32 bits, beyond the matrix up to the tile's end."""
    c = dict(M=4, N=8, K=16, groups=0, dtype=hb.BF16, a=A, lda=16, a_scale=A, w=A, ldw=16, w_scale=A, bias=0, offsets=0, y=A, ldy=8, dev_status=0)
    c.update(kw)
    m = hb.MatmulI8(*c.values())
    for call in (lambda: hb.hccl_matmul_i8(C.byref(m), 0), lambda: hb.hccl_linear_i8(C.byref(m), A, 16, hb.BF16, None, 0)):
        with pytest.raises(hb.HcclError) as e:
            call()
        assert e.value.status == hb.ERR_INVALID_ARG
