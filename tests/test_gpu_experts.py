"""Expert-layer operators on the GPU against plain 64-bit forms: routing, dispatch and combine, products in 8-bit integers."""
import numpy as np
import pytest
import torch

import expert_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SENT = 77.0


def gen(seed):
    return np.random.default_rng(seed)


def strided(t, pad=0, shift=0):
    """The same matrix on the device with `pad` more elements between rows, starting `shift` elements into its memory."""
    n, m = t.shape
    flat = torch.full((n * (m + pad) + shift + 8,), SENT, dtype=t.dtype, device="cuda")
    v = flat[shift: shift + n * (m + pad)].view(n, m + pad)[:, :m] if n else flat[:0].view(0, m + pad)[:, :m]
    v.copy_(t)
    return v


def close(got, want, tol):
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    err = np.abs(got - want)
    ok = np.isnan(want) | (err <= tol)
    assert ok.all(), (float(np.nanmax(err - tol)), int((~ok).sum()))


# ------------------------------------------------------------------------------------------------ routing
# Scores: exp of an argument rounded to 2^-24 of itself (|x| < 4 here, so 4 of them), the function's own 2 ulp, E additions, a
# division or two and the scale: within (E + 32) * 2^-24 of the weight's size, and a sum over the chosen of as much again.
def weight_tol(E, w):
    return 2 * (E + 32) * ref.EPS32 * np.abs(np.nan_to_num(w)) + 1e-37


def grid_logits(rng, T, E, dt):
    """Multiples of 1/64 in (-2, 2), exact in every type and never a pair x, -x (whose sigmoids add up to 1 in every such pair)."""
    return torch.from_numpy(((rng.integers(-31, 31, (T, E)) * 4 + 1) / 64.0).astype(np.float32)).to(dt)


ROUTES = [
    # T, E, k, score, groups, top_groups, group_best, renorm, bias, mask, dtype
    (0, 8, 2, "softmax", 1, 1, 1, True, False, False, F32),
    (1, 1, 1, "softmax", 1, 1, 1, True, False, False, BF16),
    (1, 256, 8, "sigmoid", 8, 4, 2, True, True, False, F32),
    (5, 2, 2, "sigmoid", 1, 1, 1, False, True, False, F16),
    (61, 60, 4, "softmax", 1, 1, 1, False, False, True, BF16),
    (61, 60, 6, "softmax", 4, 2, 1, True, False, True, F16),
    (300, 64, 32, "sigmoid", 1, 1, 1, True, False, False, BF16),
    (129, 320, 7, "sigmoid", 8, 3, 2, True, True, True, BF16),
    (257, 96, 5, "sigmoid", 96, 9, 1, True, True, False, F32),
    (64, 96, 3, "sigmoid", 48, 20, 2, False, False, False, F32),
    (100, 1024, 8, "softmax", 1, 1, 1, True, False, False, F32),
    (33, 1024, 16, "sigmoid", 32, 4, 2, True, True, True, F16),
    (40, 1000, 4, "softmax", 1000, 500, 1, True, False, False, F32),
    (1500, 33, 3, "softmax", 11, 4, 1, True, False, True, F32),
    (2000, 128, 8, "softmax", 1, 1, 1, True, False, False, BF16),
]


def make_route(case, seed):
    T, E, k, score, groups, top_groups, best, renorm, bias, mask, dt = case
    rng = gen(seed)
    logits = grid_logits(rng, T, E, dt)
    b = rng.integers(-2, 3, E).astype(np.float32) if bias else None
    m = (rng.random(T) < 0.8) if mask else None
    return logits, b, m, dict(groups=groups, top_groups=top_groups, group_best=best, renorm=renorm, scale=2.5)


def router_of(case):
    _, E, k, score, groups, top_groups, best, renorm, _, _, _ = case
    return ex.Router(E, k, score=score, groups=groups, top_groups=top_groups, group_best=best, renormalise=renorm, scale=2.5)


def cuda(a, dt=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def check_routing(r, ids, w, E, wtol):
    assert np.array_equal(r.ids.cpu().numpy(), ids)
    close(r.weights, w, wtol)
    counts, offsets, slots, source = ref.layout(ids, E)
    assert np.array_equal(r.counts.cpu().numpy(), counts) and np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.slots.cpu().numpy(), slots) and np.array_equal(r.source.cpu().numpy(), source)


@pytest.mark.parametrize("i", range(len(ROUTES)))
@pytest.mark.parametrize("pad", [0, 3])
def test_route_matches_the_definition(i, pad):
    case = ROUTES[i]
    logits, b, m, kw = make_route(case, 100 + i)
    ids, w, gap = ref.route(logits.float().numpy(), case[2], case[3], b, m, **kw)
    assert gap > 1e-6  # no choice hangs on rounding, so ids have to be equal
    r = router_of(case).route(strided(logits, pad, pad), cuda(b), cuda(m))
    check_routing(r, ids, w, case[1], weight_tol(case[1], w))


@pytest.mark.parametrize("T,E,k", [(20000, 256, 8), (4097, 8, 2), (30000, 60, 1), (300, 1024, 32)])
def test_layout_of_many_tokens(T, E, k):
    g = torch.Generator().manual_seed(T)
    logits = torch.randn(T, E, generator=g) + torch.linspace(2, -2, E)  # uneven experts
    r = ex.Router(E, k).route(logits.cuda())
    order = logits.sort(dim=-1, descending=True, stable=True).indices[:, :k].numpy()
    assert np.array_equal(r.ids.cpu().numpy(), order)
    flat = order.reshape(-1)
    source = np.argsort(flat, kind="stable")
    counts = np.bincount(flat, minlength=E)
    assert np.array_equal(r.source.cpu().numpy(), source) and np.array_equal(r.counts.cpu().numpy(), counts)
    assert np.array_equal(r.offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(counts)]))
    slots = np.empty(flat.size, dtype=np.int64)
    slots[source] = np.arange(flat.size)
    assert np.array_equal(r.slots.cpu().numpy().reshape(-1), slots)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("with_bias,groups", [(False, 1), (True, 1), (True, 5), (False, 5)])
def test_masked_places_and_values_that_are_not_numbers(score, dt, with_bias, groups):
    E, k = 40, 6
    rng = gen(7)
    logits = grid_logits(rng, 14, E, dt).float().numpy()
    inf, low = np.inf, float(torch.finfo(dt).min)
    logits[1] = -inf                            # nothing is left
    logits[2, 5:] = -inf                        # fewer than k are left
    logits[3] = low                             # the type's lowest value is a number: a uniform row
    logits[4, ::2] = low
    logits[5, 7] = np.nan                       # cannot be scored
    logits[6, 9] = inf                          # softmax: cannot be scored; sigmoid: 1
    logits[7] = np.nan                          # a padded token may hold anything
    logits[8] = inf
    logits[9, 3] = np.nan                       # beside an expert that is off
    logits[10, 1] = -inf
    logits[10, 2] = inf
    logits[11] = 0.0
    logits[11, ::3] = -0.0                      # both zeros are the same number
    mask = np.ones(14, dtype=np.uint8)
    mask[[7, 8]] = 0
    bias = None
    if with_bias:
        bias = rng.integers(-2, 3, E).astype(np.float32)
        bias[[3, 9, 20]] = -inf                 # rows 6 and 9 have their infinity and NaN there
    kw = dict(groups=groups, top_groups=2 if groups > 1 else 1, group_best=1, renorm=True, scale=1.0)
    ids, w, gap = ref.route(logits, k, score, bias, mask, **kw)
    assert gap > 1e-6 and (ids[1] == -1).all() and np.isnan(w[5]).all() and (ids[7:9] == -1).all()
    router = ex.Router(E, k, score=score, groups=groups, top_groups=kw["top_groups"], scale=1.0)
    lg = torch.from_numpy(logits).to(dt).cuda()
    r = router.route(lg, cuda(bias), cuda(mask).bool())
    check_routing(r, ids, w, E, weight_tol(E, w))
    # and its gradient: zeros where nothing was chosen, NaN where nothing could be scored
    dl = router.backward(lg, r, torch.ones(14, k, device="cuda"), bias=cuda(bias), token_mask=cuda(mask)).float().cpu().numpy()
    for t in range(14):
        if np.isnan(w[t]).all():
            assert np.isnan(dl[t]).all()
        else:
            assert np.isfinite(dl[t]).all()
            if (ids[t] < 0).all():
                assert (dl[t] == 0).all()


@pytest.mark.parametrize("renorm", [True, False])
def test_softmax_with_a_bias_chooses_by_the_sum(renorm):
    T, E, k = 50, 24, 5
    rng = gen(3)
    logits = grid_logits(rng, T, E, F32)
    bias = rng.integers(-1, 2, E).astype(np.float32)
    bias[4] = 1e-3
    ids, w, gap = ref.route(logits.numpy(), k, "softmax", bias, None, renorm=renorm)
    assert gap > 1e-6
    check_routing(ex.Router(E, k, renormalise=renorm).route(logits.cuda(), cuda(bias)), ids, w, E, weight_tol(E, w))


# The gradient's terms are products of three or four factors and sums of k or E of them; |dw| < 6, s <= 1, and with renormalised
# weights a division by S >= (smallest sigmoid here, 0.1): within (E + k + 64) * 2^-24 of scale * 6 / 0.1, and the output's own rounding.
@pytest.mark.parametrize("T,E,k,score,renorm,dt", [(1, 1, 1, "softmax", True, F32), (7, 8, 2, "softmax", False, F32), (61, 60, 4, "sigmoid", True, BF16),
                                                   (61, 60, 4, "sigmoid", False, F32), (300, 256, 8, "softmax", True, BF16), (64, 256, 8, "softmax", False, F16),
                                                   (33, 1024, 32, "softmax", True, F32), (2500, 128, 8, "softmax", True, BF16), (9, 33, 33 - 1, "sigmoid", True, F32)])
def test_route_gradient_matches_the_formula(T, E, k, score, renorm, dt):
    rng = gen(T + E)
    logits = grid_logits(rng, T, E, dt)
    if T > 5:
        logits[2, : E // 2] = -np.inf
        logits[3] = -np.inf
    router = ex.Router(E, k, score=score, renormalise=renorm, scale=1.5)
    lg = strided(logits, 5)
    r = router.route(lg)
    dw = np.clip(rng.standard_normal((T, k)), -5.9, 5.9).astype(np.float32)
    want = ref.route_grad(logits.double().numpy(), r.ids.cpu().numpy().astype(np.int64), dw, score, renorm, 1.5)
    out = strided(torch.full((T, E), SENT).to(dt), 2)
    got = router.backward(lg, r, cuda(dw), out=out)
    tol = (E + k + 64) * ref.EPS32 * 1.5 * 60 + ref.HALF_ULP[dt] * np.abs(want) + ref.SMALLEST[dt]
    close(got, want, tol)


@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_route_gradient_matches_differences(score, renorm):
    T, E, k, h = 40, 24, 3, 2.0 ** -7
    rng = gen(11)
    base = torch.from_numpy(np.stack([rng.permutation(E) for _ in range(T)]) / 6.0 - 2).float()  # at least 1/6 apart: +-h changes no choice
    d = torch.from_numpy(rng.uniform(-1, 1, (T, E))).float()
    dw = torch.from_numpy(rng.standard_normal((T, k))).float().cuda()
    router = ex.Router(E, k, score=score, renormalise=renorm)
    x = base.cuda().requires_grad_()
    r = router.route(x)
    (r.weights * dw).sum().backward()
    plus, minus = router.route((base + h * d).cuda()), router.route((base - h * d).cuda())
    assert torch.equal(plus.ids, r.ids) and torch.equal(minus.ids, r.ids)
    num = ((plus.weights - minus.weights).double() * dw.double()).sum(-1).cpu() / (2 * h)
    ana = (x.grad.double().cpu() * d.double()).sum(-1)
    # central differences: h^2 / 6 times a third derivative (below 8 for these functions of scores within [0, 1], along |d| <= 1, for each of
    # k weights), and the weights' rounding, 60 * 2^-24, over h
    size = dw.abs().sum(-1).double().cpu()
    assert ((num - ana).abs() <= size * (8 * h * h / 6 + 60 * ref.EPS32 / h)).all()


# ------------------------------------------------------------------------------------------------ exchange of rows
ROWS = [
    # T, k, E, H, dtype, padding between rows, shift of the base
    (0, 2, 4, 8, F32, 0, 0), (1, 1, 1, 1, BF16, 0, 0), (1, 8, 64, 4096, BF16, 0, 0), (5, 2, 4, 0, F32, 0, 0), (37, 3, 7, 89, BF16, 0, 0),
    (37, 3, 7, 90, F16, 0, 0), (64, 4, 60, 516, BF16, 4, 4), (130, 6, 60, 2056, BF16, 8, 0), (33, 32, 40, 100, F32, 1, 1), (65, 2, 8, 1030, F32, 2, 2),
    (300, 8, 16, 136, F16, 0, 8), (700, 1, 3, 24, F32, 0, 0),
]


def random_routing(T, k, E, seed, some_out=True):
    rng = gen(seed)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]) if T else np.zeros((0, k), dtype=np.int64)
    ids = ids.astype(np.int64)
    if some_out:
        ids[rng.random((T, k)) < 0.15] = -1
        if T > 2:
            ids[1] = -1
    w = rng.standard_normal((T, k)).astype(np.float32)
    w[ids < 0] = 0
    counts, offsets, slots, source = ref.layout(ids, E)
    i32 = lambda a: cuda(a.astype(np.int32))  # noqa: E731
    return ids, w, slots, source, int(offsets[-1]), ex.Routing(i32(ids), cuda(w), cuda(counts), i32(offsets), i32(slots), i32(source))


@pytest.mark.parametrize("i", range(len(ROWS)))
@pytest.mark.parametrize("short", [0, 3])
def test_dispatch_and_combine_match_the_definition(i, short):
    T, k, E, H, dt, pad, shift = ROWS[i]
    ids, w, slots, source, used, r = random_routing(T, k, E, 50 + i)
    n = max(T * k - short * max(T // 4, 1), 0)          # a capacity below the number of rows: choices are dropped
    slots = np.where(slots < n, slots, -1)
    g = torch.Generator().manual_seed(i)
    x = torch.randn(T, H, generator=g).to(dt)
    xd = x.double().numpy()
    rows_out = strided(torch.full((n, H), SENT).to(dt), pad, shift)
    got = ex.dispatch(strided(x, pad, shift), r, out=rows_out)
    want = np.zeros((n, H))
    for t, j in zip(*np.nonzero(slots >= 0)):
        want[slots[t, j]] = xd[t]
    assert np.array_equal(got.double().cpu().numpy(), want)

    rows = torch.randn(n, H, generator=g).to(dt)
    if n > used:
        rows[used:] = float("nan")                       # rows of no choice are not read
    rd = np.nan_to_num(rows.double().numpy())
    y, size, plain = np.zeros((T, H)), np.zeros((T, H)), np.zeros((T, H))
    psize = np.zeros((T, H))
    for t, j in zip(*np.nonzero(slots >= 0)):
        v = rd[slots[t, j]]
        y[t] += float(w[t, j]) * v
        size[t] += np.abs(w[t, j] * v)
        plain[t] += v
        psize[t] += np.abs(v)
    rdev = strided(rows, pad, shift)
    out = strided(torch.full((T, H), SENT).to(dt), pad, shift)
    # k products and sums in 32 bits, one rounding to the type
    close(ex.combine(rdev, r, out=out), y, (k + 1) * ref.EPS32 * size + ref.HALF_ULP[dt] * np.abs(y) * 1.01 + ref.SMALLEST[dt])
    close(ex.dispatch_backward(rdev, r), plain, (k + 1) * ref.EPS32 * psize + ref.HALF_ULP[dt] * np.abs(plain) * 1.01 + ref.SMALLEST[dt])

    dy = torch.randn(T, H, generator=g).to(dt)
    dyd = dy.double().numpy()
    drows, dw, dsize = np.zeros((n, H)), np.zeros((T, k)), np.zeros((T, k))
    for t, j in zip(*np.nonzero(slots >= 0)):
        drows[slots[t, j]] = float(w[t, j]) * dyd[t]
        dw[t, j] = dyd[t] @ rd[slots[t, j]]
        dsize[t, j] = np.abs(dyd[t] * rd[slots[t, j]]).sum()
    got_rows, got_w = ex.combine_backward(strided(dy, pad, shift), rdev, r, out=strided(torch.full((n, H), SENT).to(dt), pad, shift))
    close(got_rows, drows, (ref.HALF_ULP[dt] * 1.01 + ref.EPS32) * np.abs(drows) + ref.SMALLEST[dt])
    close(got_w, dw, (H + 2) * ref.EPS32 * dsize + 1e-37)  # H products and sums in 32 bits, in any order


def test_rows_write_nothing_beside_their_ranges():
    T, k, E, H = 50, 4, 9, 45
    ids, w, slots, source, used, r = random_routing(T, k, E, 5)
    n, pad = T * k, 7
    for dt in (F32, BF16):
        flat = torch.full((n * (H + pad) + 16,), SENT, dtype=dt, device="cuda")
        rows = flat[8: 8 + n * (H + pad)].view(n, H + pad)
        ex.dispatch(torch.ones(T, H, dtype=dt, device="cuda"), r, out=rows[:, :H])
        assert (rows[:, H:] == SENT).all() and (flat[:8] == SENT).all() and (flat[-8:] == SENT).all()
        yf = torch.full((T * (H + pad) + 16,), SENT, dtype=dt, device="cuda")
        y = yf[8: 8 + T * (H + pad)].view(T, H + pad)
        ex.combine(rows[:, :H], r, out=y[:, :H])
        assert (y[:, H:] == SENT).all() and (yf[:8] == SENT).all() and (yf[-8:] == SENT).all()


def test_offsets_beyond_32_bits():
    """Rows whose first element lies past 2^31 elements."""
    T, k, E, H = 4, 2, 2, 64
    ids, w, slots, source, used, r = random_routing(T, k, E, 1, some_out=False)
    ld = (1 << 31) // 6
    big = torch.zeros((T * k - 1) * ld + H, dtype=BF16, device="cuda")
    rows = big.as_strided((T * k, H), (ld, 1))
    x = torch.arange(T * H, dtype=F32).view(T, H).remainder(251).to(BF16).cuda()
    ex.dispatch(x, r, out=rows)
    assert torch.equal(rows[r.slots.long()], x[:, None].expand(T, k, H))
    y = ex.combine(rows, r, weights=torch.ones(T, k, device="cuda"))
    assert torch.equal(y, (2 * x.float()).to(BF16))
    q, s = ex.quantize_rows(rows)
    assert torch.equal(q[r.slots[:, 0].long()], ex.quantize_rows(x)[0])


def test_gradients_through_autograd_match_differences():
    """x -> dispatch -> rows * f -> combine with routed weights: directional differences of the whole, in 32 bits."""
    T, E, k, H, h = 30, 12, 3, 40, 2.0 ** -6
    rng = gen(2)
    base = torch.from_numpy(np.stack([rng.permutation(E) for _ in range(T)]) / 3.0 - 2).float().cuda()
    router = ex.Router(E, k)
    x0 = torch.from_numpy(rng.standard_normal((T, H))).float().cuda()
    f = torch.from_numpy(rng.standard_normal((T * k, 1))).float().cuda()
    c = torch.from_numpy(rng.standard_normal((T, H))).float().cuda()
    dx, dl = torch.randn_like(x0), torch.from_numpy(rng.uniform(-1, 1, (T, E))).float().cuda()

    def loss(x, logits):
        r = router.route(logits)
        return (ex.combine(ex.dispatch(x, r) * f, r) * c).double().sum()

    x, lg = x0.clone().requires_grad_(), base.clone().requires_grad_()
    loss(x, lg).backward()
    with torch.no_grad():
        num_x = (loss(x0 + h * dx, base) - loss(x0 - h * dx, base)) / (2 * h)
        num_l = (loss(x0, base + h * dl) - loss(x0, base - h * dl)) / (2 * h)
    size = float(T * H * 6)  # |x f c w| sums to about T * H; six times that bounds every term's share
    tol = size * 8 * ref.EPS32 / h
    assert abs(float((x.grad.double() * dx.double()).sum() - num_x)) <= tol
    assert abs(float((lg.grad.double() * dl.double()).sum() - num_l)) <= tol + size * 8 * h * h / 6
    # a gradient that arrives expanded (one row broadcast over all) is taken as it is
    r = router.route(base)
    xe = x0.clone().requires_grad_()
    ex.combine(ex.dispatch(xe, r), r).sum().backward()
    assert torch.isfinite(xe.grad).all() and xe.grad.abs().sum() > 0


# ------------------------------------------------------------------------------------------------ 8-bit rows
@pytest.mark.parametrize("M,K,dt,pad,shift", [(0, 5, F32, 0, 0), (1, 1, BF16, 0, 0), (1, 4096, BF16, 0, 0), (7, 100, F16, 3, 1), (64, 129, F32, 0, 0),
                                              (33, 8192, BF16, 8, 8), (5, 20000, F16, 0, 0), (3, 0, F32, 4, 0), (300, 1024, F32, 0, 2), (2, 131071, BF16, 0, 0)])
def test_quantised_rows_match_the_definition(M, K, dt, pad, shift):
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M + K)).to(dt)
    if M > 4:
        x[1] = 0
        x[2, K // 2] = float("nan")
        x[3, 0] = float("-inf")
        x[4] *= 1e-4 if dt == F16 else 1e-32
    q, s = ex.quantize_rows(strided(x, pad, shift))
    wq, ws = ref.quantise(x.float().numpy())
    assert np.array_equal(q.cpu().numpy(), wq)
    assert np.array_equal(s.cpu().numpy(), ws, equal_nan=True)


@pytest.mark.parametrize("T,k,E,K,dt", [(1, 8, 64, 512, BF16), (61, 3, 7, 100, F32), (200, 8, 16, 2048, F16)])
def test_quantised_dispatch_matches_quantise_then_dispatch(T, k, E, K, dt):
    ids, w, slots, source, used, r = random_routing(T, k, E, T)
    x = torch.randn(T, K, generator=torch.Generator().manual_seed(T)).to(dt)
    q, s = ex.quantize_rows(x.cuda(), routing=r)
    wq, ws = ref.quantise(x.float().numpy())
    for t, j in zip(*np.nonzero(slots >= 0)):
        assert np.array_equal(q[slots[t, j]].cpu().numpy(), wq[t]) and float(s[slots[t, j]]) == float(ws[t])


# Sums are exact; their conversion, two scales and the bias are four roundings of 2^-24, then the output's.
def product_tol(want, size, dt):
    return np.nan_to_num(4 * ref.EPS32 * size + ref.HALF_ULP[dt] * 1.01 * np.abs(want)) + ref.SMALLEST[dt]


DENSE = [(0, 8, 16), (1, 1, 1), (1, 128, 128), (1, 1000, 4096), (2, 7, 0), (3, 129, 17), (8, 256, 8192), (15, 64, 100), (16, 2048, 512), (17, 130, 129),
         (31, 513, 2064), (33, 384, 1000), (64, 1024, 1024), (65, 100, 300), (127, 257, 640), (128, 128, 128), (129, 640, 2048), (200, 96, 16), (255, 1030, 384),
         (257, 512, 4096), (300, 4104, 272), (513, 384, 1024), (1000, 777, 2000)]


@pytest.mark.parametrize("M,N,K", DENSE)
@pytest.mark.parametrize("dt,with_bias", [(BF16, False), (F32, True), (F16, True)])
def test_product_matches_the_definition(M, N, K, dt, with_bias):
    rng = gen(M * 7 + N + K)
    a, w = rng.integers(-128, 128, (M, K)).astype(np.int8), rng.integers(-128, 128, (N, K)).astype(np.int8)
    sa, sw = rng.uniform(0.5, 1.5, M).astype(np.float32) * 0.002, rng.uniform(0.5, 1.5, N).astype(np.float32) * 0.002
    b = rng.standard_normal(N).astype(np.float32) if with_bias else None
    want, size = ref.matmul(a, sa, w[None], sw[None], None if b is None else b[None])
    lin = ex.Int8Linear(cuda(w), cuda(sw), cuda(b))
    q = torch.zeros(M, (K + 15) // 16 * 16 + 16, dtype=torch.int8, device="cuda")
    q[:, K:] = 99  # what lies between rows is not part of them
    q[:, :K] = cuda(a)
    y = torch.full((M, N + 3), SENT, dtype=dt, device="cuda")
    lin.matmul(q[:, :K], cuda(sa), out=y[:, :N])
    lin.check()
    close(y[:, :N], want, product_tol(want, size, dt))
    assert (y[:, N:] == SENT).all()
    # every fourth row by itself gives the same bits: a row's result does not hang on its neighbours
    if M > 4:
        sub = lin.matmul(q[::4].contiguous()[:, :K], cuda(sa[::4].copy()), dtype=dt)
        assert torch.equal(sub, y[::4, :N])


GROUPS = [
    # N, K, rows of each group, rows before the first and after the last
    (64, 128, [0, 0, 0], 0, 5), (128, 256, [1], 0, 0), (130, 100, [3, 0, 17, 1, 0, 5], 0, 0), (256, 512, [2] * 70, 0, 3), (384, 1024, [0, 130, 0, 300, 7, 64], 4, 9),
    (200, 272, [33, 65, 1, 0, 129, 257, 2, 31], 0, 0), (2048, 1024, [9, 8, 0, 12, 3, 1, 6, 11], 0, 0), (640, 384, [700, 20], 0, 1), (96, 64, [1] * 300, 0, 0),
    (128, 2048, [1000, 0, 1, 600], 0, 0),
]


@pytest.mark.parametrize("N,K,rows,before,after", GROUPS)
@pytest.mark.parametrize("dt", [BF16, F32])
def test_product_over_groups_matches_the_definition(N, K, rows, before, after, dt):
    rng = gen(N + K + len(rows))
    G, M = len(rows), before + sum(rows) + after
    off = before + np.concatenate([[0], np.cumsum(rows)])
    a, w = rng.integers(-128, 128, (M, K)).astype(np.int8), rng.integers(-128, 128, (G, N, K)).astype(np.int8)
    sa, sw = rng.uniform(0.5, 1.5, M).astype(np.float32) * 0.002, rng.uniform(0.5, 1.5, (G, N)).astype(np.float32) * 0.002
    b = rng.standard_normal((G, N)).astype(np.float32)
    want, size = ref.matmul(a, sa, w, sw, b, off)
    lin = ex.Int8Linear(cuda(w), cuda(sw), cuda(b))
    q = torch.zeros(M, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    q[:, :K] = cuda(a)
    y = torch.full((M, N), SENT, dtype=dt, device="cuda")
    lin.matmul(q[:, :K], cuda(sa), offsets=cuda(off.astype(np.int32)), out=y)
    lin.check()
    out = np.isnan(want)
    assert (y.float().cpu().numpy()[out] == SENT).all()  # rows outside all groups are left alone
    want[out] = SENT
    close(y, want, product_tol(want, size, dt))


def test_largest_sums_are_exact():
    """K at its limit with all products at 128 * 128: the sum is just below 2^31."""
    K = hb.MAX_I8_K
    w = torch.full((3, K), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    q = torch.full((2, (K + 15) // 16 * 16), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(3, device="cuda")
    y = ex.Int8Linear(w, one).matmul(q[:, :K], one[:2], dtype=F32)
    assert y.tolist() == [[float(np.float32(16384 * K)), float(np.float32(-128 * 127 * K)), float(np.float32(16384 * K))]] * 2


@pytest.mark.parametrize("M,N,K,dt", [(1, 512, 1024, BF16), (5, 100, 77, F32), (64, 640, 512, F16), (333, 256, 2064, BF16)])
def test_linear_quantises_within_the_call(M, N, K, dt):
    g = torch.Generator().manual_seed(M)
    x = torch.randn(M, K, generator=g).to(dt)
    w = torch.randn(N, K, generator=g)
    lin = ex.Int8Linear.from_float(w.cuda())
    wq, ws = ref.quantise(w.numpy())
    xq, xs = ref.quantise(x.float().numpy())
    want, size = ref.matmul(xq, xs, wq[None], ws[None])
    y = lin(x.cuda())
    lin.check()
    close(y, want, product_tol(want, size, dt))


@pytest.mark.parametrize("T,k,E,N,K,dt", [(1, 4, 8, 256, 512, BF16), (40, 3, 9, 200, 144, F32), (64, 8, 64, 256, 256, BF16), (500, 2, 5, 384, 320, F16)])
def test_linear_over_experts_gathers_rows(T, k, E, N, K, dt):
    ids, w_, slots, source, used, r = random_routing(T, k, E, 9)
    g = torch.Generator().manual_seed(T)
    x, w = torch.randn(T, K, generator=g).to(dt), torch.randn(E, N, K, generator=g)
    lin = ex.Int8Linear.from_float(w.cuda())
    wq, ws = ref.quantise(w.numpy().reshape(-1, K))
    xq, xs = ref.quantise(x.float().numpy())
    tok = source[:used] // k
    _, offsets, _, _ = ref.layout(ids, E)
    want, size = ref.matmul(xq[tok], xs[tok], wq.reshape(E, N, K), ws.reshape(E, N), None, offsets)
    y = torch.full((T * k, N), SENT, dtype=dt, device="cuda")
    lin(x.cuda(), routing=r, out=y)
    lin.check()
    close(y[:used], want, product_tol(want, size, dt))
    assert (y[used:] == SENT).all()
    # rows that are in expert order already
    y2 = lin(ex.dispatch(x.cuda(), r), offsets=r.offsets)
    assert torch.equal(y2[:used], y[:used])


def test_rows_that_are_not_numbers_stay_in_their_row():
    x = torch.randn(20, 64).cuda()
    x[3, 5] = float("nan")
    x[7, 0] = float("inf")
    x[9] = 0
    y = ex.Int8Linear.from_float(torch.randn(40, 64).cuda())(x)
    bad = torch.zeros(20, dtype=torch.bool)
    bad[[3, 7]] = True
    assert torch.equal(torch.isnan(y).all(-1).cpu(), bad) and torch.isfinite(y[~bad.cuda()]).all() and (y[9] == 0).all()


# ------------------------------------------------------------------------------------------------ how they are used
def test_other_streams_and_repeats_give_the_same_bits():
    T, E, k, H, N = 200, 16, 4, 256, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    logits, x = torch.randn(T, E, generator=g, device="cuda"), torch.randn(T, H, generator=g, device="cuda").to(BF16)
    lin = ex.Int8Linear.from_float(torch.randn(E, N, H, generator=g, device="cuda"))
    router = ex.Router(E, k)

    def layer(lg, xx):
        r = router.route(lg)
        return ex.combine(lin(xx, routing=r), r)

    first = layer(logits, x)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = []
    for it in range(12):
        with torch.cuda.stream(streams[it % 3]):
            outs.append(layer(logits, x))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)


def test_a_whole_layer_replays_from_a_graph_with_new_inputs():
    T, E, k, H, N = 16, 8, 2, 256, 384
    g = torch.Generator(device="cuda").manual_seed(2)
    router = ex.Router(E, k, score="sigmoid")
    up, down = ex.Int8Linear.from_float(torch.randn(E, N, H, generator=g, device="cuda")), ex.Int8Linear.from_float(torch.randn(E, H, N, generator=g, device="cuda"))
    logits, x = torch.empty(T, E, device="cuda"), torch.empty(T, H, dtype=BF16, device="cuda")

    def layer(lg, xx):
        r = router.route(lg)
        return ex.combine(down(torch.relu(up(xx, routing=r)), offsets=r.offsets), r)

    logits.normal_(generator=g), x.normal_(generator=g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer(logits, x)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        y = layer(logits, x)
    for _ in range(3):
        logits.normal_(generator=g), x.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, layer(logits, x))


def test_refusals_of_the_python_layer():
    r = ex.Router(8, 2).route(torch.randn(4, 8, device="cuda"))
    lin, over = ex.Int8Linear.from_float(torch.randn(16, 32, device="cuda")), ex.Int8Linear.from_float(torch.randn(8, 16, 32, device="cuda"))
    x = torch.randn(4, 32, device="cuda")

    def refused(status, f):
        with pytest.raises(hb.HcclError) as e:
            f()
        assert e.value.status == status

    bad, mism, dty, ali = hb.ERR_INVALID_ARG, hb.ERR_COUNT_MISMATCH, hb.ERR_DTYPE, hb.ERR_ALIGNMENT
    refused(bad, lambda: ex.Router(8, 2).route(torch.randn(4, 8)))
    refused(mism, lambda: ex.Router(8, 2).route(torch.randn(4, 9, device="cuda")))
    refused(dty, lambda: ex.Router(8, 2).route(torch.randn(4, 8, device="cuda").double()))
    refused(ali, lambda: ex.Router(8, 2).route(torch.randn(8, 4, device="cuda").t()))
    refused(dty, lambda: ex.Router(8, 2).route(torch.randn(4, 8, device="cuda"), bias=torch.zeros(8, device="cuda").half()))
    refused(mism, lambda: ex.Router(8, 2).route(torch.randn(4, 8, device="cuda"), token_mask=torch.ones(3, device="cuda", dtype=torch.bool)))
    refused(mism, lambda: ex.Router(8, 2).route(torch.randn(5, 8, device="cuda"), out=r))
    refused(bad, lambda: ex.Router(8, 2).route(torch.randn(4, 8, device="cuda").requires_grad_(), out=r))
    refused(mism, lambda: ex.dispatch(torch.randn(5, 32, device="cuda"), r))
    refused(dty, lambda: ex.dispatch(x.double(), r))
    refused(dty, lambda: ex.dispatch(x, r, out=torch.empty(8, 32, device="cuda", dtype=BF16)))
    refused(mism, lambda: ex.combine(torch.randn(8, 32, device="cuda"), r, weights=torch.ones(4, 3, device="cuda")))
    refused(mism, lambda: ex.combine_backward(torch.randn(3, 32, device="cuda"), torch.randn(8, 32, device="cuda"), r))
    refused(mism, lambda: lin(torch.randn(4, 31, device="cuda")))
    refused(bad, lambda: lin(x, routing=r))
    refused(bad, lambda: over(x))
    refused(bad, lambda: over(x, routing=r, offsets=r.offsets))
    refused(mism, lambda: over(torch.randn(5, 32, device="cuda"), routing=r))
    refused(dty, lambda: over(x, offsets=r.offsets.long()))
    refused(mism, lambda: over(x, offsets=r.offsets[1:].contiguous()))
    refused(dty, lambda: lin.matmul(x, torch.ones(4, device="cuda")))
    refused(ali, lambda: lin.matmul(torch.zeros(4, 40, dtype=torch.int8, device="cuda")[:, :32], torch.ones(4, device="cuda")))
    refused(dty, lambda: ex.Int8Linear(x, torch.ones(4, device="cuda")))
    refused(mism, lambda: ex.Int8Linear(torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda")))


@pytest.mark.parametrize("M,K,dt,pad", [(4200, 4096, BF16, 0), (2100, 8192, F16, 8), (1100, 8192, F32, 4), (2100, 8184, BF16, 0), (1030, 16384, BF16, 0)])
def test_many_long_rows_quantise_alike(M, K, dt, pad):
    """Sizes that stream through shared memory: against the definition on a sample of rows, against the rows one by one on all."""
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(K)).to(dt)
    x[5] = 0
    x[M - 2, K - 1] = float("nan")
    x[M - 1, K - 1] = 900.0  # the last row's scale hangs on its last element
    xd = strided(x, pad)
    q, s = ex.quantize_rows(xd)
    pick = torch.cat([torch.arange(0, M, 97), torch.tensor([5, M - 2, M - 1])])
    wq, ws = ref.quantise(x[pick].float().numpy())
    assert np.array_equal(q[pick.cuda()].cpu().numpy(), wq) and np.array_equal(s[pick.cuda()].cpu().numpy(), ws, equal_nan=True)
    for a in range(0, M, 500):  # few rows take the other way
        q1, s1 = ex.quantize_rows(xd[a: a + 500])
        assert torch.equal(q1, q[a: a + 500]) and torch.equal(s1.view(torch.int32), s[a: a + 500].view(torch.int32))


def test_calls_captured_on_a_stream_do_not_share_scratch_with_calls_made_on_it():
    g = torch.Generator(device="cuda").manual_seed(4)
    lin = ex.Int8Linear.from_float(torch.randn(256, 512, generator=g, device="cuda"))
    a, b = (torch.randn(64, 512, generator=g, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want_a, want_b = lin(a), lin(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ya = lin(a)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(20):  # the graph on one stream, plain calls on the stream it was captured on
        with torch.cuda.stream(other):
            graph.replay()
        with torch.cuda.stream(s):
            yb = lin(b)
    torch.cuda.synchronize()
    assert torch.equal(ya, want_a) and torch.equal(yb, want_b)
