"""Expert-layer operators, host side: every refusal of the C calls comes before anything touches a device, so it is checked
here with addresses that are never followed."""
import ctypes as C

import numpy as np
import pytest

from expert_reference import layout, route
from paper_2608_00358_b200 import binding as hb

A = 1 << 20  # an aligned address that nothing reads


def status(fn, *args):
    try:
        fn(*args)
    except hb.HcclError as e:
        return e.status
    return hb.OK


def router(**kw):
    c = dict(experts=8, top_k=2, score=0, groups=1, top_groups=1, group_best=1, renormalise=1, scale=1.0)
    c.update(kw)
    return hb.RouterConfig(*c.values())


def routing(**kw):
    c = dict(tokens=4, top_k=2, experts=8, ids=A, weights=A, counts=A, offsets=A, slots=A, source=A)
    c.update(kw)
    return hb.RoutingRecord(*c.values())


@pytest.mark.parametrize("kw", [dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=9), dict(experts=64, top_k=33), dict(score=2), dict(groups=-1),
                                dict(groups=3), dict(groups=4, top_groups=0), dict(groups=4, top_groups=5), dict(groups=4, group_best=3)])
def test_router_configurations_that_do_not_hold_together(kw):
    with pytest.raises(hb.HcclError) as e:
        hb.hccl_route_workspace_bytes(router(**kw), 10)
    assert e.value.status == hb.ERR_INVALID_ARG


def test_route_workspace():
    assert hb.hccl_route_workspace_bytes(router(), 0) >= 0
    with pytest.raises(hb.HcclError):
        hb.hccl_route_workspace_bytes(router(), -1)
    with pytest.raises(hb.HcclError):
        hb.hccl_route_workspace_bytes(router(), 1 << 30)  # tokens * top_k reaches 2^31
    assert hb.hccl_route_workspace_bytes(router(), (1 << 30) - 1) < 1 << 30  # a byte for each expert and some 200 tokens


def test_route_refusals():
    n = hb.hccl_route_workspace_bytes(router(), 4) + 64

    def go(c=None, logits=A, ld=8, dt=hb.BF16, bias=0, r=None, ws=A, nbytes=n):
        return status(hb.hccl_route, C.byref(c or router()), logits, ld, dt, bias, 0, C.byref(r or routing()), ws, nbytes, 0)

    assert go(dt=3) == hb.ERR_DTYPE
    assert go(c=router(top_k=3)) == hb.ERR_COUNT_MISMATCH
    assert go(r=routing(experts=9)) == hb.ERR_COUNT_MISMATCH
    assert go(r=routing(tokens=-1)) == hb.ERR_INVALID_ARG
    assert go(logits=0) == hb.ERR_INVALID_ARG
    assert go(ld=7) == hb.ERR_INVALID_ARG
    assert go(ld=-8) == hb.ERR_INVALID_ARG
    assert go(logits=A + 1) == hb.ERR_ALIGNMENT
    assert go(bias=A + 2) == hb.ERR_ALIGNMENT
    for name in ("ids", "weights", "counts", "offsets", "slots", "source"):
        assert go(r=routing(**{name: 0})) == hb.ERR_INVALID_ARG, name
        assert go(r=routing(**{name: A + 2})) == hb.ERR_ALIGNMENT, name
    need = hb.hccl_route_workspace_bytes(router(), 4)
    assert go(nbytes=need - 1) == hb.ERR_WORKSPACE
    assert go(ws=0) == hb.ERR_INVALID_ARG
    assert go(ws=A + 4) == hb.ERR_ALIGNMENT
    back = lambda dw=A, dl=A, ldd=8: status(hb.hccl_route_backward, C.byref(router()), A, 8, hb.FP32, 0, 0, C.byref(routing()), dw, dl, ldd, 0)  # noqa: E731
    assert back(dw=0) == hb.ERR_INVALID_ARG and back(dl=0) == hb.ERR_INVALID_ARG and back(ldd=3) == hb.ERR_INVALID_ARG and back(dl=A + 2) == hb.ERR_ALIGNMENT


def test_rows_refusals():
    def disp(x=A, ldx=16, H=16, dt=hb.BF16, r=None, rows=A, ldr=16, n=8):
        return status(hb.hccl_dispatch, x, ldx, H, dt, C.byref(r or routing()), rows, ldr, n, 0)

    assert disp(dt=9) == hb.ERR_DTYPE
    assert disp(x=0) == hb.ERR_INVALID_ARG and disp(rows=0) == hb.ERR_INVALID_ARG
    assert disp(ldx=15) == hb.ERR_INVALID_ARG and disp(ldr=15) == hb.ERR_INVALID_ARG
    assert disp(H=-1) == hb.ERR_INVALID_ARG and disp(n=-1) == hb.ERR_INVALID_ARG
    assert disp(x=A + 1) == hb.ERR_ALIGNMENT
    assert disp(ldx=1 << 61) == hb.ERR_INVALID_ARG  # offsets would wrap
    assert disp(r=routing(slots=0)) == hb.ERR_INVALID_ARG and disp(r=routing(offsets=0)) == hb.ERR_INVALID_ARG
    assert disp(r=routing(top_k=33)) == hb.ERR_INVALID_ARG and disp(r=routing(tokens=1 << 30)) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_combine, A, 16, 8, 16, hb.FP32, C.byref(routing()), 0, A, 16, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_combine, A, 16, 8, 16, hb.FP32, C.byref(routing()), A + 1, A, 16, 0) == hb.ERR_ALIGNMENT
    assert status(hb.hccl_dispatch_backward, A, 16, 8, 16, hb.FP32, C.byref(routing()), 0, 16, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_combine_backward, A, 16, A, 16, 8, 16, hb.FP32, C.byref(routing()), A, A, 16, 0, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_combine_backward, A, 16, A, 16, 8, 16, hb.FP32, C.byref(routing()), A, A, 3, A, 0) == hb.ERR_INVALID_ARG


def test_quantise_refusals():
    def go(x=A, ldx=32, M=4, K=32, dt=hb.BF16, r=None, q=A, ldq=32, n=4, s=A):
        return status(hb.hccl_quantize_rows_i8, x, ldx, M, K, dt, C.byref(r) if r else None, q, ldq, n, s, 0)

    assert go(dt=7) == hb.ERR_DTYPE
    assert go(x=0) == hb.ERR_INVALID_ARG and go(q=0) == hb.ERR_INVALID_ARG and go(s=0) == hb.ERR_INVALID_ARG
    assert go(K=hb.MAX_I8_K + 1, ldx=1 << 18, ldq=1 << 18) == hb.ERR_INVALID_ARG
    assert go(ldq=31) == hb.ERR_INVALID_ARG and go(n=3) == hb.ERR_COUNT_MISMATCH
    assert go(r=routing(tokens=5), n=10) == hb.ERR_COUNT_MISMATCH
    assert go(s=A + 1) == hb.ERR_ALIGNMENT


def matmul(**kw):
    c = dict(M=4, N=8, K=32, groups=0, dtype=hb.BF16, a=A, lda=32, a_scale=A, w=A, ldw=32, w_scale=A, bias=0, offsets=0, y=A, ldy=8, dev_status=0)
    c.update(kw)
    return hb.MatmulI8(*c.values())


@pytest.mark.parametrize("kw,want", [
    (dict(M=-1), hb.ERR_INVALID_ARG), (dict(K=hb.MAX_I8_K + 1, lda=1 << 18, ldw=1 << 18), hb.ERR_INVALID_ARG), (dict(dtype=5), hb.ERR_DTYPE),
    (dict(groups=2), hb.ERR_INVALID_ARG), (dict(groups=1025, offsets=A), hb.ERR_INVALID_ARG), (dict(a=0), hb.ERR_INVALID_ARG), (dict(w=0), hb.ERR_INVALID_ARG),
    (dict(a_scale=0), hb.ERR_INVALID_ARG), (dict(w_scale=0), hb.ERR_INVALID_ARG), (dict(y=0), hb.ERR_INVALID_ARG), (dict(lda=16), hb.ERR_INVALID_ARG),
    (dict(ldw=40), hb.ERR_ALIGNMENT), (dict(lda=40), hb.ERR_ALIGNMENT), (dict(a=A + 8), hb.ERR_ALIGNMENT), (dict(w=A + 1), hb.ERR_ALIGNMENT),
    (dict(y=A + 1), hb.ERR_ALIGNMENT), (dict(ldy=7), hb.ERR_INVALID_ARG), (dict(a_scale=A + 2), hb.ERR_ALIGNMENT), (dict(bias=A + 2), hb.ERR_ALIGNMENT),
    (dict(dev_status=A + 1), hb.ERR_ALIGNMENT), (dict(M=1 << 31), hb.ERR_INVALID_ARG), (dict(N=1 << 31, ldy=1 << 31), hb.ERR_INVALID_ARG)])
def test_product_refusals(kw, want):
    m = matmul(**kw)
    assert status(hb.hccl_matmul_i8, C.byref(m), 0) == want
    assert status(hb.hccl_linear_i8, C.byref(m), A, 32, hb.BF16, None, 0) == want


def test_linear_refusals():
    m = matmul(M=8)
    assert status(hb.hccl_linear_i8, C.byref(m), 0, 32, hb.BF16, None, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_linear_i8, C.byref(m), A, 32, 4, None, 0) == hb.ERR_DTYPE
    assert status(hb.hccl_linear_i8, C.byref(m), A, 31, hb.BF16, None, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_linear_i8, C.byref(m), A, 32, hb.BF16, C.byref(routing(offsets=0)), 0) == hb.ERR_INVALID_ARG


def test_the_reference_on_a_case_worked_by_hand():
    x = np.array([[0.0, np.log(3.0), -np.inf, 0.0]])
    ids, w, _ = route(x, 3, "softmax", renorm=False)
    assert ids.tolist() == [[1, 0, 3]] and np.allclose(w, [[0.6, 0.2, 0.2]])
    counts, offsets, slots, source = layout(np.array([[1, 0], [0, -1]]), 2)
    assert counts.tolist() == [2, 1] and offsets.tolist() == [0, 2, 3] and slots.tolist() == [[2, 0], [1, -1]] and source.tolist() == [1, 2, 0, -1]
