"""Expert layers, host side: what the Python layer does before a launch, checked on the CPU with stand-ins for the device's calls."""
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
