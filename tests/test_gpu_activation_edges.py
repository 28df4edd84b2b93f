"""Gated activations on the GPU where the range ends."""
import numpy as np
import pytest
import torch

import expert_reference as eref
import fp4_reference as ref
from paper_2608_00358_b200.activation import activate, activate_backward
from test_gpu_activation import seed_of
from test_gpu_experts import BF16, F16, F32

pytestmark = pytest.mark.gpu


def near(got, want, tol, dt):
    """Within tol of a 64-bit value; infinite where that rounds to infinity, and nowhere else."""
    got = got.double().cpu().numpy()
    top = torch.finfo(dt).max
    limit = top * (1 + torch.finfo(dt).eps / 4)  # half a step above the largest number (a step is half of eps there, relative to twice the power of two)
    over, may = np.abs(want) - tol >= limit, np.abs(want) + tol >= limit
    assert not np.isnan(got).any()
    assert (got[over] == np.copysign(np.inf, want[over])).all()
    with np.errstate(invalid="ignore"):
        ok = (np.abs(got - want) <= tol) | (may & (np.isinf(got) | (np.abs(got) == top)) & (np.sign(got) == np.sign(want)))
    assert ok.all(), (got[~ok][:4], want[~ok][:4])


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
@pytest.mark.parametrize("gated", [True, False])
def test_numbers_up_to_the_types_largest(gated, p, act, dt):
    """Every product of gates, other halves and gradients, the largest numbers among them: the result's own rounding decides whether it is infinite, not what stands on the way to it."""
    top = torch.finfo(dt).max
    sizes = [0.0, 0.01, 1.0, 3.0, top / 2, 0.97 * top, top]
    gates, others, grads = (np.array([s * v for v in sizes for s in (1, -1)]) for _ in range(3))
    gates = np.concatenate([gates, [-30.0, -9.0, 0.7]])
    g, o, d = (v.ravel() for v in np.meshgrid(gates, others, grads, indexing="ij"))
    I = 56
    n = -(-g.size // I) * I
    g, o, d = (torch.from_numpy(np.resize(v, n).astype(np.float32)).clamp(-top, top).to(dt).view(-1, I) for v in (g, o, d))
    M, key = g.shape[0], (1234, 5)
    f = np.full((M, I), 1 / (1 - p)) * (ref.keep(M, I, p, key) if p else 1)
    seed = seed_of(*key) if p else None
    x = torch.cat((g, o), 1) if gated else g
    g64, o64, d64 = (v.double().numpy() for v in (g, o, d))
    with np.errstate(over="ignore"):
        a, s, _ = ref.act(act, g64)
    if not gated:
        o64 = np.ones_like(o64)

    def rounding(v):  # one of the type, and in 32 bits those of the products
        return 2.0 ** -20 * np.abs(v) + eref.HALF_ULP[dt] * np.abs(v) * 1.01 + 10 * eref.SMALLEST[dt]

    y = a * o64 * f
    near(activate(x.cuda(), act, gated, p, seed), y, rounding(y), dt)
    dx = activate_backward(d.cuda(), x.cuda(), act, gated, p, seed)
    # a slope is within 2^-20 (1 + |g|) while it changes, and 0 or 1 beyond
    dg = d64 * s * o64 * f
    near(dx[:, :I], dg, rounding(dg) + 2.0 ** -20 * np.where(np.abs(g64) < 40, 1 + np.abs(g64), 0) * np.abs(d64 * o64 * f), dt)
    assert not dx[:, :I].float().cpu().numpy()[(s == 0) | (d64 * o64 * f == 0)].any()
    if gated:
        do = d64 * a * f
        near(dx[:, I:], do, rounding(do), dt)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_silu_where_the_exponential_leaves_the_range(p, dt):
    """Gates from -91 to -86, where exp(-g) passes 2^128 and the activation is still above 2^-126: times another half or a gradient of 1e37 that is a number of order 1."""
    g = torch.linspace(-91, -86, 64).to(dt).repeat(6, 1)
    o = torch.tensor([1.0, -1.0, 1e20, 1e37, -1e37, 0.0]).to(dt)[:, None].expand(6, 64)
    d = torch.tensor([1.0, 1e30, -1.0, 1.0, 1.0, 1e37]).to(dt)[:, None].expand(6, 64)
    key = (9, 9)
    f = np.full((6, 64), 1 / (1 - p)) * (ref.keep(6, 64, p, key) if p else 1)
    seed = seed_of(*key) if p else None
    x = torch.cat((g, o), 1).cuda()
    g64, o64, d64 = (v.double().numpy() for v in (g, o, d))
    a, s, _ = ref.act("silu", g64)
    # In 32 bits exp(g) is a subnormal number: 2 units of 2^-149 off, times |g| up to 91 and another half for each of the products. Of 16-bit gates the exponential's argument, up to
    # 131, is off by 2^-17 and by what its constant's rounding leaves, and the exponential by as much.
    each = 2.0 ** -20 if dt == F32 else 2.0 ** -16
    da, ds = each * np.abs(a) + 250 * 2.0 ** -149, each * np.abs(s) + 250 * 2.0 ** -149

    def check(got, want, tol):
        tol = tol + eref.HALF_ULP[dt] * np.abs(want) * 1.01 + 2 * eref.SMALLEST[dt]
        got = got.double().cpu().numpy()
        assert (np.abs(got - want) <= tol).all(), (got[np.abs(got - want) > tol][:4], want[np.abs(got - want) > tol][:4])

    check(activate(x, "silu", True, p, seed), a * o64 * f, da * np.abs(o64) * f)
    dx = activate_backward(d.contiguous().cuda(), x, "silu", True, p, seed)
    check(dx[:, :64], d64 * s * o64 * f, ds * np.abs(d64 * o64) * f)
    check(dx[:, 64:], d64 * a * f, da * np.abs(d64) * f)
    assert (np.abs(a * 1e37) > 0.1).all()
