"""Gated activations with dropout on the GPU against 64 bits; gradients against the formula and against differences."""
import numpy as np
import pytest
import torch

import expert_reference as eref
import fp4_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex
from paper_2608_00358_b200.activation import activate, activate_backward
from test_gpu_experts import BF16, F16, F32, gen, strided
from test_gpu_fp4 import refused, routing_of, within

pytestmark = pytest.mark.gpu


def seed_of(a, b=0):
    return torch.tensor([a, b], dtype=torch.int64, device="cuda")


# An activation in 32 bits is within 2^-21 of the size of its terms (exp, erfc and a quotient: 2 ulp each, and their product), a slope within 2^-20 of its terms' (1 + |g|); then at
# most three products and one rounding to the type.
def forward(x, act, gated, f, dt):
    I = f.shape[1]
    a, _, _ = ref.act(act, x[:, :I])
    y = (a * x[:, I:] if gated else a) * f
    return y, 2.0 ** -20 * np.abs(y) + eref.HALF_ULP[dt] * np.abs(y) * 1.01 + eref.SMALLEST[dt]


def backward(dy, x, act, gated, f, dt):
    I = f.shape[1]
    g = x[:, :I]
    a, s, _ = ref.act(act, g)
    o = x[:, I:] if gated else np.ones_like(g)
    d = dy * f
    dg = d * o * s
    tol = 2.0 ** -20 * np.abs(d * o) * (1 + np.abs(g)) + eref.HALF_ULP[dt] * np.abs(dg) * 1.01 + eref.SMALLEST[dt]
    if not gated:
        return dg, tol
    do = d * a
    return np.concatenate([dg, do], 1), np.concatenate([tol, 2.0 ** -20 * np.abs(do) + eref.HALF_ULP[dt] * np.abs(do) * 1.01 + eref.SMALLEST[dt]], 1)


SIZES = [(1, 1), (1, 64), (3, 7), (40, 130), (17, 256), (130, 33), (5, 1000)]


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("act,gated,p", [("silu", True, 0.1), ("gelu", True, 0.5), ("relu", True, 0.0), ("silu", False, 0.25), ("gelu", False, 0.0), ("relu", False, 0.9)])
@pytest.mark.parametrize("M,I", SIZES)
def test_values_and_gradients(M, I, act, gated, p, dt):
    rng = gen(M + I)
    W = 2 * I if gated else I
    x = torch.from_numpy((3 * rng.standard_normal((M, W))).astype(np.float32)).to(dt)
    dy = torch.from_numpy(rng.standard_normal((M, I)).astype(np.float32)).to(dt)
    key = (-(2 ** 62) + 12345 * M, 2 ** 40 + I)
    f = np.full((M, I), 1 / (1 - p)) * (ref.keep(M, I, p, key) if p else 1)
    last = M - M // 4  # the other rows are not read and become zeros
    off = torch.tensor([0, last // 2, last], dtype=torch.int32, device="cuda")
    f_off = f.copy()
    f_off[last:] = 0
    poisoned = x.clone()
    poisoned[last:] = float("nan")
    seed = seed_of(*key) if p else None
    x64, dy64 = x.double().numpy(), dy.double().numpy()
    for shift, pad in ((0, 0), (1, 3), (8, 8)):
        xs, ds = strided(x.cuda(), pad, shift), strided(dy.cuda(), pad, shift)
        within(activate(xs, act, gated, p, seed), *forward(x64, act, gated, f, dt))
        within(activate_backward(ds, xs, act, gated, p, seed), *backward(dy64, x64, act, gated, f, dt))
        ps = strided(poisoned.cuda(), pad, shift)
        within(activate(ps, act, gated, p, seed, off), *forward(x64, act, gated, f_off, dt))
        within(activate_backward(ds, ps, act, gated, p, seed, off), *backward(dy64, x64, act, gated, f_off, dt))


def test_the_mask_is_the_same_at_every_alignment_and_differs_by_seed():
    x = torch.ones(50, 2 * 264, device="cuda")
    y = activate(x, "relu", p=0.3, seed=seed_of(5, 6))
    assert torch.equal(activate(strided(x, 1, 1), "relu", p=0.3, seed=seed_of(5, 6)), y)
    kept = (y != 0).double().mean().item()
    assert abs(kept - 0.7) < 5 * (0.21 / y.numel()) ** 0.5  # five standard deviations
    for other in (seed_of(6, 6), seed_of(5, 7), seed_of(5 + (1 << 32), 6), seed_of(5, 6 + (1 << 32))):
        assert not torch.equal(activate(x, "relu", p=0.3, seed=other), y)


def test_elements_beyond_32_bits_have_words_of_their_own():
    M, I = 70000, 65536  # 2^32 elements lie before the last rows; 9.2 GB
    x = torch.ones((M, I), dtype=BF16, device="cuda")
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    y = activate(x, "relu", gated=False, p=0.5, seed=seed_of(1, 2), offsets=off)
    row = 65536  # element 2^32 begins it
    words = []
    for n in range(row * I // 4, row * I // 4 + 16):
        words += ref.philox((n & 0xFFFFFFFF, n >> 32, 2, 0), (1, 0))
    assert ((y[row, :64] != 0).cpu().numpy() == (np.array(words) >= 2 ** 31)).all()
    assert not torch.equal(y[row], y[0])


def test_dropped_elements_are_zero_whatever_they_were():
    x = torch.full((8, 256), float("nan"), device="cuda")
    keep = ref.keep(8, 128, 0.5, (3, 4))
    y = activate(x, p=0.5, seed=seed_of(3, 4)).cpu().numpy()
    dx = activate_backward(torch.ones(8, 128, device="cuda"), x, p=0.5, seed=seed_of(3, 4)).cpu().numpy()
    assert (np.isnan(y) == keep).all() and (y[~keep] == 0).all()
    assert (np.isnan(dx) == np.concatenate([keep, keep], 1)).all()


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dt", [BF16, F16])
def test_every_16_bit_number(dt, act, p):
    """Gates of all finite 16-bit numbers: values, and both gradients, against 64 bits. In 32 bits exp(-x) is infinite below -88.73 and the activation then 0 in the place of at most 88.73 *
    2^-128 = 2.6e-37, which is what its slope leaves out too."""
    g = torch.arange(-(2 ** 15), 2 ** 15, dtype=torch.int32).to(torch.int16).view(dt)
    g = g[torch.isfinite(g.float())].reshape(-1, 64)
    if dt == BF16:
        g = g.clamp(-1e37, 1e37)  # (so that 1 / (1 - p) leaves the result in the range)
    else:
        g = g.clamp(-2e4, 2e4)
    M, I = g.shape
    x = torch.cat((g, torch.ones_like(g)), 1)
    key = (77, 78)
    f = np.full((M, I), 1 / (1 - p)) * (ref.keep(M, I, p, key) if p else 1)
    seed = seed_of(*key) if p else None
    dy = torch.ones((M, I), dtype=dt)
    x64 = x.double().numpy()
    with np.errstate(over="ignore"):  # (exp of a large negative gate: the quotient is then 0)
        y, tol = forward(x64, act, True, f, dt)
        dx, dtol = backward(dy.double().numpy(), x64, act, True, f, dt)
    within(activate(x.cuda(), act, True, p, seed), y, tol + 2.7e-37 * f)
    within(activate_backward(dy.cuda(), x.cuda(), act, True, p, seed), dx, dtol + 2.7e-37 * np.concatenate([f, f], 1))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_a_closed_gate_stays_closed_before_large_numbers(act, dt):
    g = torch.full((4, 64), -1e30, device="cuda", dtype=dt)
    x = torch.cat((g, -g), 1)
    assert not activate(x, act).any()
    assert not activate_backward(torch.full_like(g, 1e30), x, act).any()


def test_ends_of_the_range():
    for act in ("silu", "gelu", "relu"):
        g = torch.tensor([[-1e38, -200.0, -30.0, -9.0, 0.0, -0.0, 9.0, 30.0, 200.0, 1e30]], device="cuda")
        x = torch.cat((g, torch.ones_like(g)), 1)
        y, dx = activate(x, act), activate_backward(torch.ones_like(g), x, act)
        want, slope, _ = ref.act(act, np.clip(g.double().cpu().numpy(), -700, None))
        assert torch.isfinite(y).all() and torch.isfinite(dx).all()
        assert np.allclose(y.cpu().numpy(), want, rtol=2e-6, atol=1e-38) and np.allclose(dx[:, :10].cpu().numpy(), slope, rtol=1e-5, atol=2e-6)


@pytest.mark.parametrize("act,gated", [("silu", True), ("gelu", True), ("silu", False)])
def test_gradient_against_differences(act, gated):
    """Central differences of a random projection in 32 bits: the step 2^-6 leaves |f'''| h^2 / 6 < 1e-4 and 2^-22 * 64 / h < 1e-3 of rounding for sums of this size."""
    rng = gen(1)
    M, I, p, seed = 3, 20, 0.3, seed_of(9, 1)
    x = torch.from_numpy(rng.standard_normal((M, 2 * I if gated else I)).astype(np.float32)).cuda()
    dy = torch.from_numpy(rng.standard_normal((M, I)).astype(np.float32)).cuda()
    dx = activate_backward(dy, x, act, gated, p, seed)
    h = 2.0 ** -6
    for i, j in [(0, 0), (1, 3), (2, x.shape[1] - 1), (0, x.shape[1] // 2), (2, 7)]:
        a, b = x.clone(), x.clone()
        a[i, j] += h
        b[i, j] -= h
        d = ((activate(a, act, gated, p, seed).double() - activate(b, act, gated, p, seed).double()) * dy.double()).sum() / (2 * h)
        assert abs(float(d) - float(dx[i, j])) < 1e-3, (i, j)


def test_a_training_step_through_autograd():
    """dispatch, product, activation with dropout, product, combine: gradients of the tokens and of both matrices against the same step in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(3)
    T, H, I, E, k, p = 40, 48, 36, 4, 2, 0.2
    x, logits = (torch.randn(s, device="cuda", generator=g) for s in ((T, H), (T, E)))
    up, down = (torch.randn(s, device="cuda", generator=g) * s[-1] ** -0.5 for s in ((E, 2 * I, H), (E, H, I)))
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[-3:] = False
    seed = seed_of(77, 5)
    r = ex.Router(E, k).route(logits, token_mask=mask)
    off = r.offsets.tolist()
    leaves = [t.clone().requires_grad_() for t in (x, up, down)]

    def experts(rows, w):
        parts = [rows[off[e]: off[e + 1]] @ w[e].t() for e in range(E)]
        return torch.cat(parts + [rows.new_zeros(rows.shape[0] - off[E], w.shape[1])])

    rows = ex.dispatch(leaves[0], r)
    y = ex.combine(experts(activate(experts(rows, leaves[1]), p=p, seed=seed, offsets=r.offsets), leaves[2]), r)
    target = torch.randn(T, H, device="cuda", generator=g)
    (y * target).sum().backward()
    keep = torch.from_numpy(ref.keep(T * k, I, p, (77, 5))).cuda()
    ref_leaves = [t.double().requires_grad_() for t in (x, up, down)]
    token = (r.source // k).long().clamp(min=0)
    u = experts(ref_leaves[0][token], ref_leaves[1])
    h = torch.nn.functional.silu(u[:, :I]) * u[:, I:] * keep / (1 - p)
    z = experts(h, ref_leaves[2])
    w = r.weights.double() * mask[:, None]
    want = (z[r.slots.long().clamp(min=0)] * w[..., None]).sum(1)
    (want * target.double()).sum().backward()
    # sums of at most T * k terms of order 1 behind one another, in 32 bits
    for a, b in zip(leaves, ref_leaves):
        assert float((a.grad - b.grad).norm() / b.grad.norm()) < 1e-5
    assert not leaves[0].grad[-3:].any()


def test_gradients_in_any_layout_and_autograds_rules():
    x = torch.randn(6, 32, device="cuda", requires_grad=True)
    seed = seed_of(1)
    y = activate(x, p=0.1, seed=seed)
    (a,) = torch.autograd.grad(y, x, torch.ones(1, 16, device="cuda").expand(6, 16), retain_graph=True)
    (b,) = torch.autograd.grad(y, x, torch.ones(6, 16, device="cuda"), retain_graph=True)
    (c,) = torch.autograd.grad(y, x, torch.ones(16, 6, device="cuda").t(), retain_graph=True)
    assert torch.equal(a, b) and torch.equal(a, c)
    refused(hb.ERR_INVALID_ARG, lambda: activate(x, out=torch.zeros(6, 16, device="cuda")))
    seed.add_(1)
    with pytest.raises(RuntimeError):  # the mask it was made with is gone
        torch.autograd.grad(y, x, torch.ones(6, 16, device="cuda"))
    z = activate(x, p=0.0)
    (d,) = torch.autograd.grad(z.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(d.sum(), x)


def test_refusals():
    x = torch.zeros(4, 32, device="cuda")
    refused(hb.ERR_INVALID_ARG, lambda: activate(x, "tanh"))
    for p in (1.0, -0.1, float("nan"), None):
        refused(hb.ERR_INVALID_ARG, lambda: activate(x, p=p, seed=seed_of(1)))
    refused(hb.ERR_INVALID_ARG, lambda: activate(x, p=0.1))
    refused(hb.ERR_DTYPE, lambda: activate(x, p=0.1, seed=seed_of(1).int()))
    refused(hb.ERR_INVALID_ARG, lambda: activate(x, p=0.1, seed=seed_of(1).cpu()))
    refused(hb.ERR_COUNT_MISMATCH, lambda: activate(x, p=0.1, seed=seed_of(1)[:1]))
    refused(hb.ERR_COUNT_MISMATCH, lambda: activate(x[:, :31].contiguous()))
    refused(hb.ERR_COUNT_MISMATCH, lambda: activate(x, offsets=torch.zeros(1, dtype=torch.int32, device="cuda")))
    refused(hb.ERR_DTYPE, lambda: activate(x, offsets=torch.zeros(3, dtype=torch.int64, device="cuda")))
    refused(hb.ERR_DTYPE, lambda: activate(x.double()))
    refused(hb.ERR_ALIGNMENT, lambda: activate(torch.zeros(32, 4, device="cuda").t()))
    refused(hb.ERR_COUNT_MISMATCH, lambda: activate(x, out=torch.zeros(4, 17, device="cuda")))
    refused(hb.ERR_COUNT_MISMATCH, lambda: activate_backward(torch.zeros(4, 17, device="cuda"), x))
    refused(hb.ERR_DTYPE, lambda: activate_backward(torch.zeros(4, 16, device="cuda", dtype=BF16), x))
    assert activate(x[:0]).shape == (0, 16) and activate(torch.zeros(3, 0, device="cuda")).shape == (3, 0)


def test_a_captured_step_follows_its_seed():
    x = torch.randn(64, 128, device="cuda")
    seed = seed_of(10, 0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = activate(x, p=0.2, seed=seed)
        dx = activate_backward(torch.ones(64, 64, device="cuda"), x, p=0.2, seed=seed)
    for n in (1, 2):
        seed.copy_(seed_of(10, n))
        g.replay()
        assert torch.equal(y, activate(x, p=0.2, seed=seed_of(10, n)))
        assert torch.equal(dx, activate_backward(torch.ones(64, 64, device="cuda"), x, p=0.2, seed=seed_of(10, n)))
