"""Expert-layer operators where it is easy to go wrong: rows with nothing left, groups by sums of scores, scores at the ends of their range, many experts in
many groups, gradients of every layout, autograd's own rules, host threads, and the sizes at which another kernel or another turn of a loop takes over."""
import copy
import gc
import pickle
import threading
import weakref

import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

import expert_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex
from paper_2608_00358_b200.expert_layer import ExpertParallel
from test_gpu_experts import BF16, F16, F32, SENT, check_routing, close, cuda, gen, grid_logits, product_tol, random_routing, strided, weight_tol

pytestmark = pytest.mark.gpu


def refused(status, f):
    with pytest.raises(hb.HcclError) as e:
        f()
    assert e.value.status == status


# ------------------------------------------------------------------------------------------------ routing
@pytest.mark.parametrize("T,E,k,dt", [(6, 128, 3, F32), (200, 32, 3, BF16), (150, 64, 4, F32), (40, 300, 5, F32), (300, 256, 8, BF16), (33, 1024, 32, F16), (12, 12, 12, F32), (129, 128, 6, F16)])
@pytest.mark.parametrize("score,renorm,groups", [("softmax", True, 1), ("softmax", False, 1), ("softmax", True, 4), ("sigmoid", True, 1), ("sigmoid", True, 4)])
def test_rows_with_nothing_left_beside_a_bias(T, E, k, dt, score, renorm, groups):
    """Every lane of a token has experts of its own here, and all of them are out: by their logits, or by logits and bias together."""
    rng = gen(T + E)
    logits = grid_logits(rng, T, E, dt).float().numpy()
    bias = rng.integers(-2, 3, E).astype(np.float32)
    bias[1::2] = -np.inf
    logits[1] = -np.inf
    logits[4, 0::2] = -np.inf
    logits[T - 1] = -np.inf
    top_groups = groups // 2 if groups > 1 else 1
    ids, w, gap = ref.route(logits, k, score, bias, None, groups=groups, top_groups=top_groups, renorm=renorm)
    assert gap > 1e-6 and (ids[[1, 4, T - 1]] == -1).all() and (w[[1, 4, T - 1]] == 0).all()
    router = ex.Router(E, k, score=score, groups=groups, top_groups=top_groups, renormalise=renorm)
    lg = strided(torch.from_numpy(logits).to(dt), 1)
    r = router.route(lg, cuda(bias))
    check_routing(r, ids, w, E, weight_tol(E, w))
    dl = router.backward(lg, r, torch.ones(T, k, device="cuda"), bias=cuda(bias))
    assert (dl[[1, 4, T - 1]] == 0).all() and torch.isfinite(dl).all()


@pytest.mark.parametrize("bias", [False, True])
def test_two_groups_worked_by_hand(bias):
    """exp(10) + exp(-20) against 2 exp(5): the first group's scores add up to more, its logits to less."""
    logits = torch.tensor([[10.0, -20.0, 5.0, 5.0]], device="cuda")
    r = ex.Router(4, 1, groups=2, top_groups=1, group_best=2).route(logits, torch.zeros(4, device="cuda") if bias else None)
    assert r.ids.tolist() == [[0]]


@pytest.mark.parametrize("T", [2, 150])
def test_groups_far_below_the_largest_keep_their_order(T):
    """Scores that are 0 in 32 bits: the third group is the second best, the type's lowest value stands behind all other numbers, and -inf behind that."""
    low, inf = float(torch.finfo(F32).min), float("inf")
    logits = torch.tensor([[low, low, -200.0, -201.0, -150.0, -199.0, 0.0, -1.0, -inf, -inf]] * T, device="cuda")
    for groups, want in ((1, [6]), (2, [6, 4]), (3, [6, 4, 2]), (4, [6, 4, 2, 0])):
        r = ex.Router(10, 8, groups=5, top_groups=groups, group_best=2).route(logits)
        firsts = [i for i in r.ids[T - 1].tolist() if i >= 0 and i % 2 == 0]
        assert sorted(firsts) == sorted(want) and (r.ids == r.ids[0]).all()


@pytest.mark.parametrize("T,E,k,groups,top_groups,dt", [(7, 256, 8, 8, 3, BF16), (200, 96, 5, 8, 3, F32), (300, 33, 3, 11, 4, F32), (40, 320, 6, 8, 2, F16),
                                                        (150, 64, 4, 8, 3, BF16), (25, 12, 2, 4, 2, F32)])
def test_groups_under_softmax_go_by_the_sum_of_their_scores(T, E, k, groups, top_groups, dt):
    rng = gen(T + E)
    logits = grid_logits(rng, T, E, dt) * 3
    logits[1, : E // 2] = -np.inf          # groups without experts
    logits[2, 1::2] = -np.inf              # groups with half of theirs
    logits[3] = -np.inf
    # zeros for a bias: the reference's keys are the scores then, which is what a group's score is made of
    kw = dict(groups=groups, top_groups=top_groups, group_best=2, renorm=True, scale=1.0)
    ids, w, gap = ref.route(logits.float().numpy(), k, "softmax", np.zeros(E, dtype=np.float32), None, **kw)
    assert gap > 1e-6
    router = ex.Router(E, k, groups=groups, top_groups=top_groups, group_best=2)
    for bias in (None, torch.zeros(E, device="cuda")):
        r = router.route(strided(logits, 1), bias)
        assert np.array_equal(r.ids.cpu().numpy(), ids)
        close(r.weights, w, weight_tol(E, w))


@pytest.mark.parametrize("T,E,k,groups", [(9, 64, 8, 1), (300, 64, 8, 1), (40, 300, 8, 1), (200, 64, 8, 8), (10, 64, 8, 8)])
@pytest.mark.parametrize("low,high", [(10.0, 40.0), (-40.0, -10.0), (-140.0, -90.0)])
def test_sigmoid_scores_without_a_bias_choose_in_the_order_of_the_logits(T, E, k, groups, low, high):
    """Near 1 and near 0 the scores of different logits are the same number, or rounded the wrong way; the logits are not."""
    rng = gen(T)
    logits = np.stack([rng.permutation(E) for _ in range(T)]) * ((high - low) / E) + low
    logits = torch.from_numpy(logits.astype(np.float32))
    key = logits.clone()
    top_groups = max(1, groups // 2)
    if groups > 1:
        best = key.view(T, groups, -1).amax(-1).sort(dim=-1, descending=True).indices[:, :top_groups]
        keep = torch.zeros(T, groups, dtype=torch.bool).scatter_(1, best, True)
        key[~keep.repeat_interleave(E // groups, dim=1)] = -np.inf
    want = key.sort(dim=-1, descending=True, stable=True).indices[:, :k]
    r = ex.Router(E, k, score="sigmoid", groups=groups, top_groups=top_groups, renormalise=False).route(logits.cuda())
    assert torch.equal(r.ids.cpu().long(), want)
    w = 1 / (1 + np.exp(-logits.gather(1, want).double().numpy()))
    close(r.weights, w, weight_tol(E, w))


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("renorm", [True, False])
def test_a_bias_that_picks_scores_far_below_the_largest(T, renorm):
    """Renormalised weights are a softmax over the chosen: how far they lie below the others does not matter, to the weights or to their gradient."""
    E, k = 8, 2
    logits = np.tile(np.array([0.0, -150.0, -151.0, -300.0, -1.0, -2.0, -200.0, -149.0], dtype=np.float32), (T, 1))
    logits[1:] += gen(4).integers(-4, 5, (T - 1, E)).astype(np.float32) / 8
    bias = np.array([0, 4, 3, 0, 0, 0, 0, 0], dtype=np.float32)
    ids, w, gap = ref.route(logits, k, "softmax", bias, None, renorm=renorm)
    assert gap > 1e-6 and (ids == [1, 2]).all()
    router = ex.Router(E, k, renormalise=renorm)
    r = router.route(cuda(logits), cuda(bias))
    assert np.array_equal(r.ids.cpu().numpy(), ids)
    close(r.weights, w, weight_tol(E, w) + (0 if renorm else 1e-37))
    dw = gen(5).uniform(-1, 1, (T, k)).astype(np.float32)
    want = ref.route_grad(logits.astype(np.float64), ids, dw, "softmax", renorm, 1.0)
    got = router.backward(cuda(logits), r, cuda(dw), bias=cuda(bias))
    # w_j (dw_j - sum dw w): a product of two, each within (2 k + 64) 2^-24 of its terms' size, which is at most 2
    close(got, want, (2 * k + 64) * ref.EPS32 * 2 + ref.HALF_ULP[F32] * np.abs(want) + 1e-37)


@pytest.mark.parametrize("k", [2, 5])
@pytest.mark.parametrize("E", [16, 300])
def test_gradient_of_renormalised_sigmoids_near_zero(E, k):
    """Scores of 1e-38 with a gradient of some hundreds (a scaled loss): 1 / S times the gradient leaves the range, the result does not."""
    T = 20
    rng = gen(E)
    logits = (-86.0 + np.stack([rng.permutation(E) for _ in range(T)]) / E).astype(np.float32)
    dw = rng.uniform(-300, 300, (T, k)).astype(np.float32)
    router = ex.Router(E, k, score="sigmoid")
    r = router.route(cuda(logits))
    want = ref.route_grad(logits.astype(np.float64), r.ids.cpu().numpy().astype(np.int64), dw, "sigmoid", True, 1.0)
    got = router.backward(cuda(logits), r, cuda(dw))
    # scores at the lower end of the normal numbers: exp within 2 ulp, sums and quotients of k of them, terms up to 2 * 300
    close(got, want, (2 * k + 64) * ref.EPS32 * 600 + ref.HALF_ULP[F32] * np.abs(want))


@pytest.mark.parametrize("T", [9, 15, 16, 31, 32, 33])
@pytest.mark.parametrize("k", [8, 32])
@pytest.mark.parametrize("E", [1024, 990])
def test_as_many_groups_as_experts(T, k, E):
    g = torch.Generator().manual_seed(T)
    logits = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() / 64
    r = ex.Router(E, k, groups=E, top_groups=E // 2).route(logits.cuda())
    order = logits.sort(dim=-1, descending=True).indices[:, :k]
    assert torch.equal(r.ids.cpu().long(), order)
    counts, offsets, slots, source = ref.layout(order.numpy(), E)
    assert np.array_equal(r.slots.cpu().numpy(), slots) and np.array_equal(r.source.cpu().numpy(), source) and np.array_equal(r.offsets.cpu().numpy(), offsets)


# ------------------------------------------------------------------------------------------------ host threads
def test_host_threads_on_one_stream_do_not_share_scratch():
    """Two threads that call the same router and the same layer on the default stream, with rows and token counts of their own."""
    E, k, K, N = 16, 4, 256, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    router, lin = ex.Router(E, k), ex.Int8Linear.from_float(torch.randn(E, N, K, generator=g, device="cuda"))
    sizes = (700, 3001)
    logits, x = [torch.randn(T, E, generator=g, device="cuda") for T in sizes], [torch.randn(T, K, generator=g, device="cuda") for T in sizes]
    want = []
    for i in range(2):
        r = router.route(logits[i])
        want.append((r, lin(x[i], routing=r)))
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(2)

    def work(i):
        start.wait()
        for turn in range(150):
            r = router.route(logits[i])
            y = lin(x[i], routing=r)
            if turn % 10 == 9 and not (torch.equal(r.source, want[i][0].source) and torch.equal(r.slots, want[i][0].slots) and torch.equal(y, want[i][1])):
                wrong.append((i, turn))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


# ------------------------------------------------------------------------------------------------ the layer over ranks
def test_an_expert_layer_takes_any_stride_and_refuses_other_shapes():
    R, k, tokens, hidden, inner = 3, 2, 20, 48, 32
    g = torch.Generator(device="cuda").manual_seed(0)
    up, down = [[ex.Int8Linear.from_float(torch.randn(1, n, m, device="cuda", generator=g)) for _ in range(R)] for n, m in ((inner, hidden), (hidden, inner))]
    layer = ExpertParallel(ex.Router(R, k), up, down, tokens)
    x, logits = [torch.randn(tokens, hidden, device="cuda", generator=g) for _ in range(R)], [torch.randn(tokens, R, device="cuda", generator=g) for _ in range(R)]
    want = layer.forward(x, logits)
    layer.check()
    got = layer.forward([strided(t, 5, 3) for t in x], logits)
    layer.check()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    mism, bad, ali, dty = hb.ERR_COUNT_MISMATCH, hb.ERR_INVALID_ARG, hb.ERR_ALIGNMENT, hb.ERR_DTYPE
    for status, t in ((mism, x[0][:-1]), (mism, x[0][:, :-1]), (ali, torch.randn(hidden, tokens, device="cuda").t()), (bad, x[0].cpu()), (dty, x[0].double()), (bad, x[0][0])):
        refused(status, lambda: layer.forward([x[0], t, x[2]], logits))
    refused(mism, lambda: layer.forward(x[:2], logits))
    refused(bad, lambda: layer.forward([x[0], x[1], x[2].clone().requires_grad_()], logits))
    refused(mism, lambda: layer.forward(x, logits[:2]))
    refused(mism, lambda: layer.forward(x, [logits[0][:-1], logits[1], logits[2]]))
    refused(mism, lambda: ExpertParallel(ex.Router(R, k), up[:2], down, tokens))
    refused(mism, lambda: ExpertParallel(ex.Router(R, k), up, up, tokens))
    assert all(torch.equal(a, b) for a, b in zip(layer.forward(x, logits), want))


# ------------------------------------------------------------------------------------------------ gradients and autograd
@pytest.mark.parametrize("T", [0, 1, 12])
@pytest.mark.parametrize("H", [1, 5, 64])
@pytest.mark.parametrize("how", ["sum", "sum over tokens", "mean over tokens", "sum over columns", "transposed"])
def test_gradients_arrive_in_any_layout(T, H, how):
    k, E = 3, 6
    r = random_routing(T, k, E, 3)[-1]
    g = torch.Generator(device="cuda").manual_seed(H)
    c = torch.randn(H, generator=g, device="cuda")

    def loss(y):
        if how == "sum":
            return y.sum()
        if how == "sum over tokens":
            return (y.sum(0) * c).sum()
        if how == "mean over tokens":
            return (y.mean(0) * c).sum()
        if how == "sum over columns":
            return (y.sum(1) ** 2).sum()
        return (y.t().contiguous() * c[:, None]).sum()

    def grad_of(y):
        z = y.detach().requires_grad_()
        loss(z).backward()
        return z.grad.contiguous()

    x = torch.randn(T, H, generator=g, device="cuda").requires_grad_()
    rows = ex.dispatch(x, r)
    loss(rows).backward()
    assert torch.equal(x.grad, ex.dispatch_backward(grad_of(rows), r))
    v = torch.randn(T * k, H, generator=g, device="cuda").requires_grad_()
    w = torch.randn(T, k, generator=g, device="cuda").requires_grad_()
    y = ex.combine(v, r, weights=w)
    loss(y).backward()
    want_v, want_w = ex.combine_backward(grad_of(y), v.detach(), r, weights=w.detach())
    assert torch.equal(v.grad, want_v) and torch.equal(w.grad, want_w)


def test_second_derivatives_are_refused():
    T, E, k, H = 6, 8, 2, 16
    router = ex.Router(E, k)
    logits, x = torch.randn(T, E, device="cuda").requires_grad_(), torch.randn(T, H, device="cuda").requires_grad_()
    r = router.route(logits)
    plain = router.route(logits.detach())
    v = torch.randn(T * k, H, device="cuda").requires_grad_()
    for out, by in (((r.weights ** 2).sum(), logits), ((ex.dispatch(x, plain) ** 2).sum(), x), ((ex.combine(v, plain) ** 2).sum(), v)):
        d, = torch.autograd.grad(out + (by ** 3).sum(), by, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):  # not a Hessian of the second term alone
            (d ** 2).sum().backward()


def test_forward_mode_is_refused():
    T, E, k, H = 6, 8, 2, 32
    router, lin = ex.Router(E, k), ex.Int8Linear.from_float(torch.randn(16, H, device="cuda"))
    logits, x, v, w = (torch.randn(s, device="cuda") for s in ((T, E), (T, H), (T * k, H), (T, k)))
    r = router.route(logits)
    bad = hb.ERR_INVALID_ARG
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        refused(bad, lambda: router.route(dual(logits)))
        refused(bad, lambda: router.route(dual(logits), out=r))
        refused(bad, lambda: router.backward(dual(logits), r, w))
        refused(bad, lambda: router.backward(logits, r, dual(w)))
        refused(bad, lambda: ex.dispatch(dual(x), r))
        refused(bad, lambda: ex.dispatch_backward(dual(v), r))
        refused(bad, lambda: ex.combine(dual(v), r))
        refused(bad, lambda: ex.combine(v, r, weights=dual(w)))
        refused(bad, lambda: ex.combine_backward(dual(x), v, r))
        refused(bad, lambda: ex.combine_backward(x, dual(v), r))
        refused(bad, lambda: lin(dual(x)))
        refused(bad, lambda: ex.quantize_rows(dual(x)))
        assert torch.equal(ex.dispatch(x, r), ex.dispatch(x.clone(), r))  # what has no tangent goes through


def test_a_linear_layer_without_a_gradient_says_so():
    lin = ex.Int8Linear.from_float(torch.randn(16, 32, device="cuda"))
    x = torch.randn(4, 32, device="cuda").requires_grad_()
    refused(hb.ERR_INVALID_ARG, lambda: lin(x))
    refused(hb.ERR_INVALID_ARG, lambda: ex.quantize_rows(x))
    q, scale = ex.quantize_rows(x.detach())
    refused(hb.ERR_INVALID_ARG, lambda: lin.matmul(q, scale.clone().requires_grad_()))
    with torch.no_grad():
        y = lin(x)
    assert torch.equal(y, lin(x.detach())) and not y.requires_grad


def test_a_layer_is_made_from_parameters():
    w, b = torch.nn.Parameter(torch.randn(24, 40, device="cuda")), torch.nn.Parameter(torch.randn(24, device="cuda"))
    x = torch.randn(5, 40, device="cuda")
    y = ex.Int8Linear.from_float(w, b)(x)
    assert not y.requires_grad and torch.equal(y, ex.Int8Linear.from_float(w.detach(), b.detach())(x))


def test_writes_through_out_are_seen_by_autograd():
    T, E, k, H = 10, 8, 2, 32
    router, lin = ex.Router(E, k), ex.Int8Linear.from_float(torch.randn(16, H, device="cuda"))
    logits, x, v, w = (torch.randn(s, device="cuda") for s in ((T, E), (T, H), (T * k, H), (T, k)))
    r = router.route(logits)

    def bumped(tensors, call):
        before = [t._version for t in tensors]
        call()
        assert all(t._version > b for t, b in zip(tensors, before))

    bumped([r.ids, r.weights, r.counts, r.offsets, r.slots, r.source], lambda: router.route(logits, out=r))
    dl, y, dx, rows, lo = torch.empty_like(logits), torch.empty_like(x), torch.empty_like(x), torch.empty_like(v), torch.empty(T, 16, device="cuda")
    q, s = ex.quantize_rows(x)
    bumped([dl], lambda: router.backward(logits, r, w, out=dl))
    bumped([rows], lambda: ex.dispatch(x, r, out=rows))
    bumped([dx], lambda: ex.dispatch_backward(v, r, out=dx))
    bumped([y], lambda: ex.combine(v, r, out=y))
    bumped([rows], lambda: ex.combine_backward(x, v, r, out=rows))
    bumped([lo], lambda: lin(x, out=lo))
    bumped([lo], lambda: lin.matmul(q, s, out=lo))
    # a buffer that autograd holds: torch refuses the gradient
    p = torch.ones(T, 1, device="cuda").requires_grad_()
    z = y * p
    ex.combine(v, r, out=y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()
    with torch.inference_mode():
        buf = torch.empty(T, H, device="cuda")
        ex.combine(v, r, out=buf)
        router.route(logits, out=router.outputs(T))
    ex.combine(v, r, out=buf)  # has no version to count
    # an output that is part of a graph itself
    refused(hb.ERR_INVALID_ARG, lambda: ex.combine(v, r, out=torch.empty(T, H, device="cuda").requires_grad_()))
    refused(hb.ERR_INVALID_ARG, lambda: router.route(logits, out=router.route(logits.clone().requires_grad_())))
    with torch.no_grad():
        ex.combine(v, r, out=torch.empty(T, H, device="cuda").requires_grad_())


@pytest.mark.parametrize("T,E", [(1, 8), (32, 1024), (128, 64), (129, 64), (33, 1024), (17, 200)])
def test_calls_that_need_no_workspace_touch_none(T, E):
    """Up to some 128 tokens one block does everything; the workspace it is given stays as it was, whichever call that is."""
    logits = torch.randn(T, E, device="cuda")
    router = ex.Router(E, 2)
    out = router.outputs(T)
    need = hb.hccl_route_workspace_bytes(router.config, T)
    assert need >= hb.ROUTE_NO_WORKSPACE
    ws = torch.full((need,), 0xa5, dtype=torch.uint8, device="cuda")
    ex._route(router._at, logits.data_ptr(), E, hb.FP32, 0, 0, out.at, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert (need == hb.ROUTE_NO_WORKSPACE) == bool((ws == 0xa5).all())
    r = router.route(logits)
    assert torch.equal(r.source, out.source) and torch.equal(r.weights, out.weights)


@pytest.mark.parametrize("what", ["dispatch", "combine"])
def test_a_routing_that_is_routed_into_again_refuses_its_gradient(what):
    T, E, k, H = 10, 8, 2, 32
    router = ex.Router(E, k)
    a, b = torch.randn(T, E, device="cuda"), torch.randn(T, E, device="cuda")
    r = router.outputs(T)
    x, v = torch.randn(T, H, device="cuda").requires_grad_(), torch.randn(T * k, H, device="cuda").requires_grad_()

    def forward():
        return ex.dispatch(x, r) if what == "dispatch" else ex.combine(v, r, weights=torch.ones(T, k, device="cuda"))

    router.route(a, out=r)
    forward().sum().backward()  # in order: nothing to refuse
    y = forward()
    router.route(b, out=r)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_training_step_leaves_nothing_for_the_collector():
    router, logits = ex.Router(16, 2), torch.randn(40, 16, device="cuda").requires_grad_()
    gc.collect()
    gc.disable()
    try:
        for step in ("with backward", "without"):
            r = router.route(logits)
            held = [weakref.ref(t) for t in (r.ids, r.weights, r.source)]
            if step == "with backward":
                (r.weights ** 2).sum().backward()
            del r
            assert [h() for h in held] == [None] * 3, step
    finally:
        gc.enable()


def test_layers_of_one_thread_share_their_scratch():
    K, N, M = 2048, 64, 4096
    lins = [ex.Int8Linear.from_float(torch.randn(N, K, device="cuda")) for _ in range(4)]
    x, y = torch.randn(M, K, device="cuda"), torch.empty(M, N, device="cuda")
    want = [lin(x) for lin in lins]
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for lin in lins:
        lin(x, out=y)
    more = [ex.Int8Linear(lin.weight, lin.scale) for lin in lins]
    got = [lin(x) for lin in more]
    assert torch.cuda.memory_allocated() - before < 4 * (M * N * 4 + 1024)  # the results and the status words, no rows in 8 bits
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_copies_have_addresses_of_their_own():
    logits, x, w = torch.randn(9, 8, device="cuda"), torch.randn(9, 40, device="cuda"), torch.randn(8, 24, 40, device="cuda")
    router, lin = ex.Router(8, 3, score="sigmoid", groups=4, top_groups=2, group_best=2, renormalise=False, scale=2.5), ex.Int8Linear.from_float(w, torch.randn(8, 24, device="cuda"))
    r = router.route(logits)
    y = lin(x, routing=r)
    used = int(r.offsets[-1])
    for make in (copy.copy, copy.deepcopy, lambda o: pickle.loads(pickle.dumps(o))):
        router2, lin2 = make(router), make(lin)
        assert router2._at != router._at and router2.config is not router.config
        if make is not copy.copy:
            assert lin2.weight.data_ptr() != lin.weight.data_ptr() and lin2._fixed[0] == lin2.weight.data_ptr()
        r2 = router2.route(logits)
        assert torch.equal(r2.ids, r.ids) and torch.equal(r2.weights, r.weights)
        assert torch.equal(lin2(x, routing=r2)[:used], y[:used])
    r3 = copy.deepcopy(r)
    assert r3.slots.data_ptr() != r.slots.data_ptr() and r3.record.slots == r3.slots.data_ptr()
    assert torch.equal(lin(x, routing=r3)[:used], y[:used])


# ------------------------------------------------------------------------------------------------ other kernels, other turns of their loops
@pytest.mark.parametrize("T,k,E,H,dt,pad,short", [(300, 8, 40, 1032, BF16, 0, 0), (300, 8, 40, 1032, BF16, 8, 37), (130, 32, 60, 2056, F16, 16, 11), (1200, 2, 9, 4100, F32, 4, 0),
                                                  (5000, 4, 16, 136, F32, 0, 100), (40, 3, 7, 24584, BF16, 0, 0)])
def test_dispatch_of_many_bytes(T, k, E, H, dt, pad, short):
    """From 4 MB of rows on, by bulk copies: rows of several pieces with a remainder, distances between rows, places without a row, a capacity that drops some,
    a tail without choices. Nothing but copies: equal bits, and nothing beside the rows' ranges."""
    es = torch.empty(0, dtype=dt).element_size()
    assert T * k * H * es >= 4 << 20 and H * es % 16 == 0 and (H + pad) * es % 16 == 0
    ids, w, slots, source, used, r = random_routing(T, k, E, T)
    n = (used - short) if short else T * k
    assert short or n > used  # either some choices are dropped or a tail is left
    x = torch.randn(T, H, generator=torch.Generator().manual_seed(k)).to(dt)
    flat = torch.full((n * (H + pad) + 64,), SENT, dtype=dt, device="cuda")
    out = flat[32: 32 + n * (H + pad)].view(n, H + pad)
    ex.dispatch(strided(x, pad), r, out=out[:, :H])
    want = torch.zeros(n, H, dtype=dt)
    t, j = np.nonzero((slots >= 0) & (slots < n))
    want[torch.from_numpy(slots[t, j])] = x[torch.from_numpy(t)]
    assert torch.equal(out[:, :H].cpu(), want)
    assert (out[:, H:] == SENT).all() and (flat[:32] == SENT).all() and (flat[-32:] == SENT).all()


@pytest.mark.parametrize("M,N,K,dt", [(2000, 2900, 384, BF16), (5000, 1030, 272, F32), (600, 16400, 128, F16), (20000, 512, 1024, BF16)])
def test_pairs_of_blocks_walk_several_tiles(M, N, K, dt):
    """More tiles of 256 x 256 than there are pairs of SMs: accumulators and stages in turn, the last tile ragged."""
    assert -(-M // 256) * -(-N // 256) > 74
    g = torch.Generator(device="cuda").manual_seed(M)
    a = torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-127, 128, (N, K), generator=g, device="cuda").to(torch.int8)
    sa, sw = torch.rand(M, generator=g, device="cuda") * 0.002 + 0.001, torch.rand(N, generator=g, device="cuda") * 0.002 + 0.001
    lin = ex.Int8Linear(w, sw)
    y = torch.full((M, N + 1), SENT, dtype=dt, device="cuda")
    lin.matmul(a, sa, out=y[:, :N])
    lin.check()
    want = (a.double() @ w.double().t()) * sa.double()[:, None] * sw.double()  # sums below 2^53: exact
    want = want.cpu().numpy()
    close(y[:, :N], want, product_tol(want, np.abs(want), dt))
    assert (y[:, N:] == SENT).all()


@pytest.mark.parametrize("M,N,K,dt", [(2, 300, 8192, BF16), (3, 100, 5000, F32), (8, 512, 4096, BF16), (8, 130, 8200, F16), (5, 64, 13000, F16), (8, 48, 20000, BF16)])
def test_few_long_rows_are_quantised_ahead(M, N, K, dt):
    """Few rows that are too long for every block to quantise: the quantiser, and the product of few rows behind it; the last too long for that one too."""
    assert M * K > 8192
    g = torch.Generator().manual_seed(K)
    x, w = torch.randn(M, K, generator=g).to(dt), torch.randn(N, K, generator=g)
    lin = ex.Int8Linear.from_float(w.cuda())
    wq, ws = ref.quantise(w.numpy())
    xq, xs = ref.quantise(x.float().numpy())
    want, size = ref.matmul(xq, xs, wq[None], ws[None])
    for _ in range(3):
        y = lin(x.cuda())
    lin.check()
    close(y, want, product_tol(want, size, dt))


@pytest.mark.parametrize("T,E,k,score", [(80000, 24, 3, "softmax"), (200000, 8, 2, "sigmoid"), (18900, 1024, 4, "softmax"), (600000, 5, 1, "softmax")])
def test_layout_of_chunks_that_count_by_other_rules(T, E, k, score):
    """Chunks of more than 63 tokens (from 75 777 on), and more chunks than a line adds up at once (1024 experts, some 18 900 tokens)."""
    g = torch.Generator().manual_seed(T)
    mask = torch.rand(T, generator=g) < 0.9
    logits = (torch.rand(T, E, generator=g) * 4 - 2 + torch.linspace(1, -1, E)).float()
    r = ex.Router(E, k, score=score).route(logits.cuda(), token_mask=mask.cuda())
    order = logits.sort(dim=-1, descending=True, stable=True).indices[:, :k].numpy()
    order[~mask.numpy()] = -1
    flat = order.reshape(-1)
    live = np.nonzero(flat >= 0)[0]
    source = np.full(flat.size, -1)
    source[: live.size] = live[np.argsort(flat[live], kind="stable")]
    slots = np.full(flat.size, -1)
    slots[source[: live.size]] = np.arange(live.size)
    counts = np.bincount(flat[live], minlength=E)
    assert np.array_equal(r.ids.cpu().numpy(), order) and np.array_equal(r.counts.cpu().numpy(), counts)
    assert np.array_equal(r.offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(counts)]))
    assert np.array_equal(r.source.cpu().numpy(), source) and np.array_equal(r.slots.cpu().numpy().reshape(-1), slots)


def row_scaled_gradient(logits, ids, dw, score, renorm, scale, bias=None):
    """The gradient in 64 bits by its formula, and the size of the terms of each element."""
    off = np.isneginf(logits) | (np.zeros(logits.shape, dtype=bool) if bias is None else np.isneginf(bias)[None])
    with np.errstate(all="ignore"):
        top = np.where(off, -np.inf, logits).max(-1, keepdims=True)
        e = np.where(off, 0.0, np.exp(logits - top))
        s = np.where(off, 0.0, 1 / (1 + np.exp(-logits))) if score == "sigmoid" else e / np.maximum(e.sum(-1, keepdims=True), 1e-300)
    live = ids >= 0
    at = np.where(live, ids, 0)
    c = np.where(live, np.take_along_axis(s, at, 1), 0.0)
    g = np.where(live, dw * float(scale), 0.0)
    if renorm:
        total = c.sum(-1, keepdims=True)
        p = np.where(total > 0, c / np.where(total > 0, total, 1.0), 0.0)
        d, size = p * (g - (g * p).sum(-1, keepdims=True)), p * (np.abs(g) + (np.abs(g) * p).sum(-1, keepdims=True))
        if score == "sigmoid":
            d = d * (1 - c)
    elif score == "sigmoid":
        d, size = g * c * (1 - c), np.abs(g) * c
    if renorm or score == "sigmoid":
        D, S = np.zeros(s.shape), np.zeros(s.shape)
        t, j = np.nonzero(live)
        D[t, ids[t, j]], S[t, ids[t, j]] = d[t, j], size[t, j]
        return D, S
    G = np.zeros(s.shape)
    t, j = np.nonzero(live)
    G[t, ids[t, j]] = g[t, j]
    return s * (G - (G * s).sum(-1, keepdims=True)), s * (np.abs(G) + (np.abs(G) * s).sum(-1, keepdims=True))


@pytest.mark.parametrize("T,E,k,score,renorm,dt,with_bias", [
    (50, 320, 8, "softmax", False, F32, False), (33, 1024, 32, "softmax", False, F32, True), (40, 300, 5, "softmax", True, F32, True), (33, 1024, 32, "softmax", True, F32, False),
    (25, 1000, 6, "sigmoid", True, F32, True), (25, 1000, 6, "sigmoid", False, BF16, True), (61, 60, 4, "softmax", False, F16, True), (300, 256, 8, "softmax", True, BF16, True),
    (200, 128, 8, "sigmoid", True, F32, True), (40000, 16, 2, "softmax", True, F32, False), (40000, 12, 2, "softmax", False, BF16, True), (20000, 260, 2, "softmax", False, F32, False)])
def test_route_gradient_within_the_size_of_its_terms(T, E, k, score, renorm, dt, with_bias):
    """Scores in 32 bits are within (E + 32) 2^-24 of themselves (the sum over E of them), a dot of k terms within (k + 8) 2^-24 of theirs, then a few roundings: within
    (2 E + 2 k + 64) 2^-24 of the size of an element's own terms, and the output's rounding."""
    rng = gen(T + E + k)
    logits = grid_logits(rng, T, E, dt)
    logits[2, : E // 2] = -np.inf
    logits[3] = -np.inf
    bias = None
    if with_bias:
        bias = rng.integers(-1, 2, E).astype(np.float32)
        bias[[1, E // 3]] = -np.inf
    router = ex.Router(E, k, score=score, renormalise=renorm, scale=1.5)
    lg = strided(logits, 3)
    r = router.route(lg, cuda(bias))
    ids = r.ids.cpu().numpy().astype(np.int64)
    assert (ids[3] == -1).all() and (bias is None or not np.isin(ids, [1, E // 3]).any())
    dw = np.clip(rng.standard_normal((T, k)), -5.9, 5.9).astype(np.float32)
    want, size = row_scaled_gradient(logits.double().numpy(), ids, dw, score, renorm, 1.5, bias)
    got = router.backward(lg, r, cuda(dw), bias=cuda(bias))
    close(got, want, (2 * E + 2 * k + 64) * ref.EPS32 * size + ref.HALF_ULP[dt] * 1.01 * np.abs(want) + ref.SMALLEST[dt] + 1e-37)


@pytest.mark.parametrize("seed", range(4))
def test_random_routers(seed):
    """60 configurations: experts, groups, scores, biases and masks of every kind, rows with -inf, NaN and infinities in them; routing, layout and gradient. A row whose choice hangs
    on less than 1e-6 is left out of the comparison of choices."""
    rng = gen(900 + seed)
    pick = lambda *a: a[rng.integers(len(a))]  # noqa: E731
    compared = 0
    for _ in range(60):
        E = int(pick(rng.integers(1, 65), rng.integers(1, 401), 2 ** rng.integers(3, 11), rng.integers(200, 1025)))
        groups = int(pick(1, 1, pick(*[d for d in range(1, E + 1) if E % d == 0])))
        top_groups, best, k = int(rng.integers(1, groups + 1)), int(pick(1, 2)), int(rng.integers(1, min(32, E) + 1))
        T = min(int(pick(rng.integers(1, 21), rng.integers(1, 301), rng.integers(100, 1501))), max(1, 100000 // E))
        score, renorm, dt = pick("softmax", "sigmoid"), bool(rng.integers(2)), pick(F32, BF16, F16)
        logits = (grid_logits(rng, T, E, dt) * int(pick(1, 2))).float().numpy()
        for t in range(T):
            u = rng.random()
            if u < 0.2:
                logits[t, rng.random(E) < pick(0.5, 0.95, 1.0)] = -np.inf
            elif u < 0.25:
                logits[t, rng.integers(E)] = pick(np.nan, np.inf)
        bias = None
        if rng.integers(2):
            bias = rng.integers(-2, 3, E).astype(np.float32)
            bias[rng.random(E) < pick(0.0, 0.1, 0.5, 0.95)] = -np.inf
        mask = (rng.random(T) < 0.8) if rng.integers(2) else None
        # (zeros for a bias where group scores are sums: the reference's keys are the scores then)
        bias_ref = np.zeros(E, dtype=np.float32) if bias is None and score == "softmax" and groups > 1 and best == 2 else bias
        ids, w, sure = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k)), np.ones(T, dtype=bool)
        for t in range(T):
            i, v, gap = ref.route(logits[t: t + 1], k, score, bias_ref, None if mask is None else mask[t: t + 1], groups=groups, top_groups=top_groups, group_best=best, renorm=renorm, scale=2.5)
            ids[t], w[t], sure[t] = i[0], v[0], gap > 1e-6
        compared += int(sure.sum())
        what = (T, E, k, score, groups, top_groups, best, renorm, dt, bias is not None)
        router = ex.Router(E, k, score=score, groups=groups, top_groups=top_groups, group_best=best, renormalise=renorm, scale=2.5)
        lg = strided(torch.from_numpy(logits).to(dt), int(pick(0, 0, 3, 4)), int(pick(0, 1, 4)))
        r = router.route(lg, cuda(bias), cuda(mask))
        got, got_w = r.ids.cpu().numpy().astype(np.int64), r.weights.double().cpu().numpy()
        assert np.array_equal(got[sure], ids[sure]), what
        close(r.weights[torch.from_numpy(sure).cuda()], w[sure], weight_tol(E, w[sure]))
        for a, b in zip((r.counts, r.offsets, r.slots, r.source), ref.layout(got, E)):
            assert np.array_equal(a.cpu().numpy(), b), what
        dw = np.clip(rng.standard_normal((T, k)), -5.9, 5.9).astype(np.float32)
        dl = router.backward(lg, r, cuda(dw), bias=cuda(bias), token_mask=cuda(mask))
        unscored = np.isnan(got_w).any(-1)
        live = ~unscored & (np.ones(T, dtype=bool) if mask is None else mask)
        x = np.where(np.isposinf(logits), 800.0, logits).astype(np.float64)  # (a sigmoid of 1)
        want, size = row_scaled_gradient(x, np.where(live[:, None], got, -1), dw, score, renorm, 2.5, bias)
        chose = live & (got >= 0).any(-1)
        want[~chose], size[~chose] = 0, 0
        want[unscored] = np.nan
        close(dl, want, (2 * E + 2 * k + 64) * ref.EPS32 * np.nan_to_num(size) + ref.HALF_ULP[dt] * 1.01 * np.abs(np.nan_to_num(want)) + ref.SMALLEST[dt] + 1e-37)
    assert compared > 1000
