"""Gated activations on the GPU where the range ends, and where a thread has many rows."""
import numpy as np
import pytest
import torch

import expert_reference as eref
import fp4_reference as ref
from paper_2608_00358_b200.activation import activate, activate_backward
from test_gpu_activation import seed_of
from test_gpu_experts import BF16, F16, F32, strided

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


# ------------------------------------------------------------------------------------------------ threads that walk from row to row
def words(n, key):
    """The first n words of the generator, on the device."""
    M32 = 0xFFFFFFFF

    def product(a, m):  # high and low half, a below 2^32
        lo = a * (m & 0xFFFF)
        mid = a * (m >> 16) + (lo >> 16)
        return mid >> 16, ((mid & 0xFFFF) << 16) | (lo & 0xFFFF)

    at = torch.arange(-(-n // 4), device="cuda")
    c = [at & M32, at >> 32, torch.full_like(at, key[1] & M32), torch.full_like(at, (key[1] >> 32) & M32)]
    k = [key[0] & M32, (key[0] >> 32) & M32]
    for _ in range(10):
        (h0, l0), (h1, l1) = product(c[0], 0xD2511F53), product(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k[0], l1, h0 ^ c[3] ^ k[1], l0]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return torch.stack(c, -1).flatten()[:n]


def test_the_words_on_the_device_are_those_of_the_reference():
    key = (-(2 ** 61) - 99, 2 ** 45 + 7)
    assert (words(1002, key).cpu().numpy() >= 2 ** 31).tolist() == ref.keep(1, 1002, 0.5, key)[0].tolist()


@pytest.mark.parametrize("M,I,p,gated,act,dt", [
    # 148 * 12 blocks at most with dropout, 148 * 64 without, of 4 rows (up to 32 pieces of 16 bytes in a row) to 1: each thread has three rows or more, or some two
    (16000, 40, 0.1, True, "silu", BF16), (80000, 24, 0.0, True, "gelu", F16), (12001, 33, 0.3, True, "relu", F32), (90000, 9, 0.0, False, "silu", F32),
    (5000, 1504, 0.25, True, "gelu", BF16), (20000, 1100, 0.0, False, "silu", BF16), (21000, 1280, 0.0, True, "silu", F16), (4000, 999, 0.1, True, "silu", F32),  # two pieces of a row
    (4000, 3000, 0.1, True, "gelu", F32), (3000, 6200, 0.5, False, "gelu", F16), (3600, 5000, 0.2, True, "relu", BF16),  # more pieces than are on their way at once
])
def test_rows_one_after_the_other(M, I, p, gated, act, dt):
    """Every element of value and gradient against 64 bits where a thread goes on from row to row, with rows that are read no further than the last expert's, and at other alignments."""
    g = torch.Generator(device="cuda").manual_seed(M + I)
    W = 2 * I if gated else I
    x, dy = (2 * torch.randn((M, W), device="cuda", generator=g)).to(dt), torch.randn((M, I), device="cuda", generator=g).to(dt)
    key, last = (M * 2 ** 33 + 5, -I), M - M // 3 - 1
    f = torch.full((M, I), 1 / (1 - p), dtype=torch.float64, device="cuda")
    if p:
        f *= (words(M * I, key) >= round(p * 2.0 ** 32)).view(M, I)
    seed = seed_of(*key) if p else None
    g64, o64, d64 = x[:, :I].double(), x[:, I:].double() if gated else 1.0, dy.double()
    if act == "silu":
        s = torch.sigmoid(g64)
        a, slope = g64 * s, s * (1 + g64 * (1 - s))
    elif act == "gelu":
        phi = 0.5 * torch.special.erfc(-g64 * 0.5 ** 0.5)
        a, slope = g64 * phi, phi + g64 * torch.exp(-0.5 * g64 * g64) * (0.5 / np.pi) ** 0.5
    else:
        a, slope = g64.clamp(min=0), (g64 > 0).double()
    off = torch.tensor([0, last // 3, last], dtype=torch.int32, device="cuda")
    for shift, pad, offsets in ((0, 0, None), (0, 0, off), (8, 8, off), (1, 3, off)):
        if offsets is not None:
            f[last:] = 0
            x[last:] = float("nan")
        half, least = eref.HALF_ULP[dt] * 1.01, eref.SMALLEST[dt]

        def check(got, want, tol):
            want, tol = (torch.where(f == 0, 0.0, v) for v in (want, tol))  # (what is dropped, and rows that are not read: 0)
            assert ((got.double() - want).abs() <= tol + half * want.abs() + least).all(), (shift, pad)

        y = a * o64 * f
        xs, ds = strided(x, pad, shift), strided(dy, pad, shift)
        check(activate(xs, act, gated, p, seed, offsets), y, 2.0 ** -20 * y.abs())
        dx = activate_backward(ds, xs, act, gated, p, seed, offsets)
        check(dx[:, :I], d64 * slope * o64 * f, 2.0 ** -20 * (d64 * o64 * f).abs() * (1 + g64.abs()))
        if gated:
            do = d64 * a * f
            check(dx[:, I:], do, 2.0 ** -20 * do.abs())
