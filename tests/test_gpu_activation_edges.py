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
