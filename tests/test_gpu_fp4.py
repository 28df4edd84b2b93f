"""Operators in 4-bit floating point on the GPU: rows against the definition bit for bit, products and the layer for few tokens against 64 bits."""
import copy
import pickle
import threading

import numpy as np
import pytest
import torch

import expert_reference as eref
import fp4_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex
from paper_2608_00358_b200 import fp4
from test_gpu_experts import BF16, F16, F32, SENT, gen, strided

pytestmark = pytest.mark.gpu
FORMATS = ("nvfp4", "mxfp4")


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def refused(status, f):
    with pytest.raises(hb.HcclError) as e:
        f()
    assert e.value.status == status


def within(got, want, tol):
    half = got.dtype == F16
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    err = np.abs(got - want)
    ok = np.isnan(want) | (err <= tol)
    if half:  # from 65520 on, half a step above its largest number, fp16 rounds to infinity
        ok |= np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + tol >= 65520)
    assert ok.all(), (float(np.nanmax(err - tol)), int((~ok).sum()))


def routing_of(ids, E, w=None):
    """A Routing of given ids (numpy, -1: none)."""
    counts, offsets, slots, source = eref.layout(ids, E)
    w = np.ones(ids.shape, dtype=np.float32) if w is None else w
    return ex.Routing(cuda(ids.astype(np.int32)), cuda(w.astype(np.float32)), cuda(counts), cuda(offsets.astype(np.int32)), cuda(slots.astype(np.int32)), cuda(source.astype(np.int32)))


def some_ids(rng, T, k, E, none=0.0):
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]) if T else np.zeros((0, k), dtype=np.int64)
    return np.where(rng.random(ids.shape) < none, -1, ids)


# ------------------------------------------------------------------------------------------------ rows
def awkward(rng, M, K):
    """Rows with what can go wrong: ties, zeros, infinities, NaN, the smallest and largest numbers."""
    x = rng.standard_normal((M, K)).astype(np.float32) * np.exp2(rng.integers(-12, 12, (M, 1))).astype(np.float32)
    for m in range(M):
        kind = m % 8
        if kind == 1:
            x[m] = np.rint(x[m] * 8) / 8  # many ties
        elif kind == 2:
            x[m, rng.integers(0, K, max(1, K // 40))] = np.inf
            x[m, rng.integers(0, K)] = -np.nan
        elif kind == 3:
            x[m] = 0
            x[m, K // 2:] = -0.0
        elif kind == 4:
            x[m] *= np.float32(1e-38)  # subnormal for a part
        elif kind == 5:
            x[m, ::3] = 3e38
        elif kind == 6:
            x[m, rng.random(K) < 0.9] = 0
    return x


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("fmt,wide", [("nvfp4", 1.0), ("nvfp4", 0.0173), ("nvfp4", 3e-30), ("mxfp4", 1.0)])
@pytest.mark.parametrize("M,K,pad,shift", [(1, 1, 0, 0), (9, 15, 1, 0), (16, 64, 0, 0), (33, 257, 3, 1), (24, 512, 8, 8), (10, 1040, 0, 0), (17, 4095, 0, 0)])
def test_rows_bit_for_bit(M, K, pad, shift, fmt, wide, dt):
    x = torch.from_numpy(awkward(gen(M + K), M, K)).to(dt)
    codes, scale = ref.quantise(x.float().numpy(), fmt, wide)
    rows = fp4.quantize_rows(strided(x.cuda(), pad, shift), fmt, wide)
    assert np.array_equal(rows.scale.cpu().numpy(), scale)
    assert np.array_equal(rows.q.cpu().numpy(), ref.pack(codes))
    want = torch.from_numpy(ref.values(codes, scale, fmt, wide).astype(np.float32))  # a product of at most 6 and 24 bits, rounded once
    for out_dt in (F32, BF16, F16):
        got, ref_dt = rows.dequantize(out_dt), want.to(out_dt)
        assert torch.equal(torch.nan_to_num(got.cpu().float(), 12345.0), torch.nan_to_num(ref_dt.float(), 12345.0))
    out = strided(torch.zeros(M, K), 5, 1)
    rows.dequantize(out=out)
    assert torch.equal(torch.nan_to_num(out.cpu()), torch.nan_to_num(want))


def test_no_rows_and_no_columns():
    for shape in ((0, 64), (5, 0), (0, 0)):
        rows = fp4.quantize_rows(torch.zeros(shape, device="cuda"))
        assert rows.dequantize(BF16).shape == shape


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,K,E,k,none", [(1, 64, 4, 1, 0), (70, 200, 8, 3, 0.2), (33, 1024, 60, 6, 0)])
def test_rows_in_expert_order(T, K, E, k, none, fmt):
    rng = gen(T)
    x = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).to(BF16)
    ids = some_ids(rng, T, k, E, none)
    r = routing_of(ids, E)
    codes, scale = ref.quantise(x.float().numpy(), fmt)
    source = r.source.cpu().numpy()
    n = int((source >= 0).sum())
    for cap in (T * k, max(n - 3, 0), T * k + 5):
        rows = fp4.quantize_rows(x.cuda(), fmt, routing=r, n_rows=cap)
        m = min(n, cap)
        t = source[:m] // k
        assert rows.q.shape[0] == cap
        assert np.array_equal(rows.q[:m].cpu().numpy(), ref.pack(codes)[t]) and np.array_equal(rows.scale[:m].cpu().numpy(), scale[t])


def test_rows_that_no_choice_fills_are_left_alone():
    r = routing_of(np.array([[0, -1], [1, 0]]), 2)
    x = torch.ones(2, 64, device="cuda", dtype=BF16)
    q, s = torch.full((6, 32), 99, dtype=torch.uint8, device="cuda"), torch.full((6, 4), 99, dtype=torch.uint8, device="cuda")
    hb.hccl_quantize_rows_fp4(x.data_ptr(), 64, 2, 64, hb.BF16, hb.NVFP4, 1.0, hb.C.byref(r.record), q.data_ptr(), 32, s.data_ptr(), 4, 6, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (q[:3] != 99).all() and (q[3:] == 99).all() and (s[:3] != 99).all() and (s[3:] == 99).all()


def test_rows_beyond_32_bits_of_offset():
    M, K = 140000, 32768  # 9.2 GB of input, 2.3 GB of codes: both pass 2^31
    x = torch.zeros((M, K), dtype=BF16, device="cuda")
    tail = torch.randn((3, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(BF16)
    x[-3:] = tail
    rows = fp4.quantize_rows(x)
    want = fp4.quantize_rows(tail)
    assert torch.equal(rows.q[-3:], want.q) and torch.equal(rows.scale[-3:], want.scale) and not rows.q[:-3].any()
    del x
    got = rows.dequantize(BF16)
    assert torch.equal(got[-3:], want.dequantize(BF16)) and not got[-4].any()


def test_rows_that_overlap_are_refused():
    one = fp4.quantize_rows(torch.ones(1, 64, device="cuda"))
    rows = fp4.Fp4Rows(one.q.expand(5, -1), one.scale.expand(5, -1), 64)
    refused(hb.ERR_INVALID_ARG, rows.dequantize)
    wide = torch.zeros(5, 48, dtype=torch.uint8, device="cuda")
    wide[:, :32], scales = one.q, one.scale.repeat(5, 3)
    got = fp4.Fp4Rows(wide[:, :32], scales[:, :4], 64).dequantize()  # rows further apart than they are long
    assert torch.equal(got, one.dequantize().expand(5, -1))


# ------------------------------------------------------------------------------------------------ products
# Sums in 32 bits: an instruction adds 64 products (exact) to the accumulator, each aligned to the largest of them and cut at its last bit: within K * 2^-23 of the
# sum of the terms' sizes; then the factor, the bias (2^-24 each) and the type's rounding.
def product(values, w, factor, bias, dt):
    y = (values @ w.T) * factor
    size = (np.abs(values) @ np.abs(w).T) * factor
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    K = values.shape[1]
    return y, (K + 4) * 2.0 ** -23 * size + eref.HALF_ULP[dt] * np.abs(y) * 1.01 + eref.SMALLEST[dt]


def make_linear(rng, shape, fmt, bias, x_scale=1.0):
    flat, scale, values = ref.weights(rng, shape, fmt)
    G = shape[0] if len(shape) == 3 else 1
    wide = (0.5 + rng.random(G)).astype(np.float32) if fmt == "nvfp4" else np.ones(G, dtype=np.float32)
    b = rng.standard_normal(shape[:-1]).astype(np.float32) * 100 if bias else None
    lin = fp4.Fp4Linear(cuda(flat), cuda(scale), cuda(wide), format=fmt, bias=None if b is None else cuda(b), x_scale=x_scale, K=shape[-1])
    return lin, values.reshape((G,) + values.shape[-2:]), wide.astype(np.float64), None if b is None else b.reshape(G, -1).astype(np.float64)


DENSE = [
    # M, N, K, dtype of x and y, bias: one for each tile (16 to 256 tokens), clusters that share K, ragged edges
    (1, 1, 1, BF16, False), (1, 128, 64, F32, True), (1, 2048, 4096, BF16, False), (3, 130, 65, F16, True), (8, 512, 2048, F32, False), (16, 640, 320, BF16, True),
    (17, 129, 257, F32, True), (33, 1024, 1024, F16, False), (64, 384, 4096, F32, True), (65, 200, 96, BF16, False), (128, 4096, 512, BF16, True), (129, 127, 1000, F32, False),
    (256, 2048, 768, BF16, False), (300, 1030, 515, F16, True), (777, 2304, 256, BF16, False), (1025, 515, 288, F32, True),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K,dt,bias", DENSE)
def test_dense_product(M, N, K, dt, bias, fmt):
    rng = gen(M + N + K)
    x_scale = 0.0173 if fmt == "nvfp4" else 1.0
    lin, w, wide, b = make_linear(rng, (N, K), fmt, bias, x_scale)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(dt)
    want, tol = product(ref.rounded(x.float().numpy(), fmt, x_scale) , w[0], wide[0], None if b is None else b[0], dt)
    y = lin(strided(x.cuda(), 3, 1))
    within(y, want, tol)
    out = strided(torch.full((M, N), SENT), 7, 1).to(dt) if dt != F32 else strided(torch.full((M, N), SENT), 7, 1)
    assert lin(x.cuda(), out=out) is out
    assert torch.equal(out, y)
    assert torch.equal(lin.matmul(fp4.quantize_rows(x.cuda(), fmt, x_scale), dtype=dt), y)
    lin.check()


GROUPED = [(1, 8, 1, 130, 64, BF16), (5, 4, 2, 128, 257, F32), (40, 8, 2, 256, 512, BF16), (300, 16, 4, 200, 320, F16), (900, 3, 2, 384, 288, BF16), (2000, 5, 3, 136, 160, F32), (64, 60, 6, 129, 1024, BF16)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,E,k,N,K,dt", GROUPED)
def test_product_over_experts(T, E, k, N, K, dt, fmt):
    rng = gen(T + N)
    lin, w, wide, b = make_linear(rng, (E, N, K), fmt, T % 2 == 1)
    x = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).to(dt)
    ids = some_ids(rng, T, k, E, 0.1)
    ids[ids == E - 1] = 0  # an expert without rows; a token may have one twice
    r = routing_of(ids, E)
    values = ref.rounded(x.float().numpy(), fmt)
    offsets, source = r.offsets.cpu().numpy(), r.source.cpu().numpy()
    n = offsets[-1]
    want, tol = np.full((T * k, N), SENT), np.zeros((T * k, N))
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:
            want[lo:hi], tol[lo:hi] = product(values[source[lo:hi] // k], w[e], wide[e], None if b is None else b[e], dt)
    out = torch.full((T * k, N), SENT, dtype=dt, device="cuda")
    lin(x.cuda(), routing=r, out=out)
    within(out, want, tol)  # rows behind the last expert's are as they were
    out2 = torch.full((T * k, N), SENT, dtype=dt, device="cuda")
    lin(ex.dispatch(x.cuda(), r), offsets=r.offsets, out=out2)
    assert torch.equal(out2, out)
    out3 = torch.full((T * k, N), SENT, dtype=dt, device="cuda")
    lin.matmul(fp4.quantize_rows(x.cuda(), fmt, routing=r), offsets=r.offsets, out=out3)
    assert torch.equal(out3[:n], out[:n]) and (out3[n:] == SENT).all()
    lin.check()


@pytest.mark.parametrize("lo,hi", [(5, 6), (2, 4), (0, 1)])
@pytest.mark.parametrize("T,K", [(9, 136), (700, 264)])
def test_product_of_a_share_of_a_larger_routing(T, K, lo, hi):
    """Some of the experts, with the offsets of all choices' rows: the share's rows against 64 bits, the others left alone."""
    rng = gen(15)
    E, k, N = 6, 2, 72
    some, w, wide, _ = make_linear(rng, (hi - lo, N, K), "nvfp4", False)
    x = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).to(BF16).cuda()
    r = routing_of(some_ids(rng, T, k, E), E)
    share = ex.Routing(r.ids, r.weights, r.counts[lo:hi].clone(), r.offsets[lo:hi + 1].clone(), r.slots, r.source)
    values, offsets, source = ref.rounded(x.float().cpu().numpy(), "nvfp4"), r.offsets.cpu().numpy(), r.source.cpu().numpy()
    want, tol = np.full((T * k, N), SENT), np.zeros((T * k, N))
    for e in range(lo, hi):
        a, b = offsets[e], offsets[e + 1]
        want[a:b], tol[a:b] = product(values[source[a:b] // k], w[e - lo], wide[e - lo], None, F32)
    rows = fp4.quantize_rows(x, routing=r)
    for f in (lambda out: some(x, routing=share, out=out), lambda out: some.matmul(rows, offsets=share.offsets, out=out),
              lambda out: some(ex.dispatch(x, r), offsets=share.offsets, out=out)):
        out = torch.full((T * k, N), SENT, dtype=F32, device="cuda")
        f(out)
        within(out, want, tol)
    some.check()


def test_product_with_nothing_to_do():
    lin, _, _, _ = make_linear(gen(0), (64, 128), "nvfp4", True)
    assert lin(torch.zeros(0, 128, device="cuda", dtype=BF16)).shape == (0, 64)
    none = fp4.Fp4Linear(torch.zeros((8, 0), dtype=torch.uint8, device="cuda"), torch.zeros((8, 0), dtype=torch.uint8, device="cuda"), bias=torch.arange(8.0, device="cuda"))
    assert torch.equal(none(torch.zeros(3, 0, device="cuda")), torch.arange(8.0, device="cuda").expand(3, 8))


@pytest.mark.parametrize("fmt", FORMATS)
def test_infinities_and_nan_stay_in_their_rows(fmt):
    rng = gen(3)
    lin, w, wide, _ = make_linear(rng, (256, 300), fmt, False)
    x = rng.standard_normal((40, 300)).astype(np.float32)
    x[3, 5], x[17, 299], x[39, 0] = np.nan, np.inf, -np.inf
    want, tol = product(ref.rounded(x, fmt), w[0], wide[0], None, F32)
    assert np.isnan(want[[3, 17, 39]]).all() and np.isnan(want).sum() == 3 * 256
    within(lin(cuda(x)), want, tol)


@pytest.mark.parametrize("fmt", FORMATS)
def test_from_float_and_back(fmt):
    rng = gen(4)
    w = rng.standard_normal((3, 70, 130)).astype(np.float32)
    lin = fp4.Fp4Linear.from_float(torch.nn.Parameter(cuda(w)), format=fmt)
    wide = [float(v) for v in lin.tensor_scale]
    x = torch.eye(128, 130, device="cuda") * 4
    four = ref.rounded(np.array([[4.0]]), fmt)[0, 0]  # 4 is 6 x 0.6875 = 4.125 in "nvfp4": 4 / 6 is no e4m3 number
    assert four == (4.125 if fmt == "nvfp4" else 4.0)
    for e in range(3):
        off = torch.zeros(4, dtype=torch.int32, device="cuda")
        off[e + 1:] = 128
        got, want = lin(x, offsets=off).cpu().numpy().T, four * ref.rounded(w[e], fmt, wide[e])[:, :128]
        # one product each: the step's rounding in the reference, the factor's, the sum's (exact) and the result's
        assert (np.abs(got - want) <= 3 * 2.0 ** -24 * np.abs(want)).all()
        if fmt == "nvfp4":
            assert wide[e] == np.float32(np.float32(np.abs(w[e]).max()) / np.float32(2688))


def test_linear_refusals():
    q, s = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 4), dtype=torch.uint8, device="cuda")
    lin = fp4.Fp4Linear(q, s)
    x = torch.zeros(2, 64, device="cuda")
    refused(hb.ERR_DTYPE, lambda: fp4.Fp4Linear(q, s, format="fp4"))
    refused(hb.ERR_DTYPE, lambda: fp4.Fp4Linear(q.float(), s))
    refused(hb.ERR_DTYPE, lambda: fp4.Fp4Linear(q.view(torch.int8), s))
    refused(hb.ERR_COUNT_MISMATCH, lambda: fp4.Fp4Linear(q, s, format="mxfp4"))
    refused(hb.ERR_COUNT_MISMATCH, lambda: fp4.Fp4Linear(q, s, K=62))
    refused(hb.ERR_COUNT_MISMATCH, lambda: fp4.Fp4Linear(q, s, torch.ones(2, device="cuda")))
    refused(hb.ERR_INVALID_ARG, lambda: fp4.Fp4Linear(q.cpu(), s))
    refused(hb.ERR_INVALID_ARG, lambda: fp4.Fp4Linear(q, s.cpu()))
    for bad in (0.0, -1.0, float("nan"), 1e31, None):
        refused(hb.ERR_INVALID_ARG, lambda: fp4.Fp4Linear(q, s, x_scale=bad))
        refused(hb.ERR_INVALID_ARG, lambda: fp4.quantize_rows(x, scale=bad))
    refused(hb.ERR_COUNT_MISMATCH, lambda: lin(x[:, :63]))
    refused(hb.ERR_DTYPE, lambda: lin(x.double()))
    refused(hb.ERR_INVALID_ARG, lambda: lin(x, offsets=torch.zeros(2, dtype=torch.int32, device="cuda")))
    refused(hb.ERR_INVALID_ARG, lambda: lin(x.clone().requires_grad_()))
    refused(hb.ERR_INVALID_ARG, lambda: fp4.quantize_rows(x.clone().requires_grad_()))
    refused(hb.ERR_ALIGNMENT, lambda: lin(torch.zeros(64, 2, device="cuda").t()))
    refused(hb.ERR_DTYPE, lambda: lin.matmul(fp4.quantize_rows(x, "mxfp4")))
    refused(hb.ERR_COUNT_MISMATCH, lambda: lin.matmul(fp4.quantize_rows(x[:, :62])))
    refused(hb.ERR_DTYPE, lambda: fp4.quantize_rows(x).dequantize(torch.float64))
    over = fp4.Fp4Linear(q[None], s[None])
    refused(hb.ERR_INVALID_ARG, lambda: over(x))
    refused(hb.ERR_COUNT_MISMATCH, lambda: over(x, offsets=torch.zeros(3, dtype=torch.int32, device="cuda")))


def test_one_byte_types_of_torch_and_weights_of_any_layout():
    rng = gen(5)
    flat, scale, w = ref.weights(rng, (40, 96), "nvfp4")
    x = torch.from_numpy(rng.standard_normal((5, 96)).astype(np.float32)).cuda()
    want = fp4.Fp4Linear(cuda(flat), cuda(scale))(x)
    assert torch.equal(fp4.Fp4Linear(cuda(flat), cuda(scale).view(torch.float8_e4m3fn))(x), want)
    wide = torch.zeros((40, 60), dtype=torch.uint8, device="cuda")
    wide[:, 3:51], view = cuda(flat), wide[:, 3:51]
    assert torch.equal(fp4.Fp4Linear(view, cuda(scale).t().contiguous().t())(x), want)


@pytest.mark.parametrize("how", ["copy", "deepcopy", "pickle"])
def test_copies_have_addresses_of_their_own(how):
    f = {"copy": copy.copy, "deepcopy": copy.deepcopy, "pickle": lambda v: pickle.loads(pickle.dumps(v))}[how]
    rng = gen(6)
    up, _, _, _ = make_linear(rng, (4, 64, 33), "nvfp4", True, 0.5)
    down, _, _, _ = make_linear(rng, (4, 33, 32), "nvfp4", False)
    few = fp4.FewTokens(up, down, "gelu")
    x = torch.randn(3, 33, device="cuda")
    r = routing_of(some_ids(rng, 3, 2, 4), 4)
    want, y = up(x, routing=r), few(x, r)
    rows = fp4.quantize_rows(x)
    up2, few2, rows2 = f(up), f(few), f(rows)
    del up, few
    assert torch.equal(up2(x, routing=r), want) and torch.equal(few2(x, r), y) and torch.equal(rows2.dequantize(), rows.dequantize())


# ------------------------------------------------------------------------------------------------ the layer for few tokens
def layer_reference(x, ids, weights, up, down, act, gated, fmt, dt):
    """y in 64 bits and a bound of the error: of the pieces (2^-22 of a row's largest element, for each weight), of the sums (2^-23 for each term), of the
    activation (its slope; a few steps of its own), and the type's rounding."""
    wu, gu, bu = up
    wd, gd, bd = down
    left = 2.0 ** -22
    T, H = x.shape
    I = wd.shape[-1]

    def linear(v, dv, w, g, b):
        y, mag = w @ v * g, np.abs(w) @ np.abs(v) * g
        if b is not None:
            y, mag = y + b, mag + np.abs(b)
        top = np.abs(v).max() if v.size else 0.0
        return y, np.abs(w) @ dv * g + np.abs(w).sum(1) * g * left * top + (len(v) + 40) * 2.0 ** -23 * mag

    y, tol = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for j, e in enumerate(ids[t]):
            if e < 0:
                continue
            u, du = linear(x[t], np.zeros(H), wu[e], gu[e], None if bu is None else bu[e])
            a, _, steep = ref.act(act, u[:I])
            da = steep * du[:I] + 2.0 ** -20 * (np.abs(a) + np.abs(u[:I]) * 2.0 ** -2)
            h, dh = (a * u[I:], da * np.abs(u[I:]) + np.abs(a) * du[I:] + da * du[I:]) if gated else (a, da)
            z, dz = linear(h, dh, wd[e], gd[e], None if bd is None else bd[e])
            y[t] += weights[t, j] * z
            tol[t] += abs(weights[t, j]) * (dz + 2.0 ** -20 * np.abs(z))
    return y, tol + eref.HALF_ULP[dt] * np.abs(y) * 1.01 + eref.SMALLEST[dt]


LAYERS = [
    # T, H, I, E, k, act, gated, bias, none, dtype
    (1, 1, 1, 1, 1, "silu", True, False, 0, F32), (1, 64, 32, 4, 2, "silu", True, False, 0, BF16), (1, 1024, 512, 16, 8, "silu", True, True, 0, F32),
    (2, 257, 129, 3, 3, "gelu", True, True, 0, F16), (3, 300, 70, 5, 2, "relu", False, True, 0.3, F32), (9, 512, 300, 2, 2, "silu", True, False, 0, F32),
    (17, 136, 65, 4, 3, "gelu", False, False, 0.2, BF16), (33, 640, 104, 8, 4, "silu", True, True, 0.1, F32), (64, 260, 130, 6, 5, "silu", True, False, 0, F32),
    (64, 96, 48, 1, 1, "silu", True, False, 0, F16), (5, 2050, 1030, 7, 2, "silu", True, True, 0, F32), (4, 64, 64, 1024, 4, "silu", True, False, 0, F32),
    (64, 40, 24, 32, 32, "silu", True, False, 0, F32), (64, 33, 17, 1024, 32, "relu", False, True, 0, F32),  # as many rows as there can be, in few chunks and in many
    (7, 48, 2100, 5, 2, "silu", True, False, 0, F32), (2, 4100, 40, 6, 6, "gelu", True, False, 0, BF16),  # many parts on one side, one on the other
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,H,I,E,k,act,gated,bias,none,dt", LAYERS)
def test_layer_for_few_tokens(T, H, I, E, k, act, gated, bias, none, dt, fmt):
    rng = gen(T + H + I)
    up, wu, gu, bu = make_linear(rng, (E, (2 if gated else 1) * I, H), fmt, bias)
    down, wd, gd, bd = make_linear(rng, (E, H, I), fmt, bias)
    # outputs of order 1: by the matrices' own scales, which both formats take as they are
    for lin, n in ((up, H), (down, I)):
        lin.tensor_scale.mul_(1 / (np.sqrt(n) * 150 if fmt == "nvfp4" else np.sqrt(n) / 4))
    gu, gd = up.tensor_scale.double().cpu().numpy(), down.tensor_scale.double().cpu().numpy()
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32) * np.exp2(rng.integers(-3, 4, H)).astype(np.float32)).to(dt)
    ids = some_ids(rng, T, k, E, none)
    w = rng.random((T, k)).astype(np.float32)
    r = routing_of(ids, E, w)
    few = fp4.FewTokens(up, down, act, gated)
    want, tol = layer_reference(x.double().numpy(), ids, w.astype(np.float64), (wu, gu, bu), (wd, gd, bd), act, gated, fmt, dt)
    y = few(strided(x.cuda(), 3, 1), r)
    within(y, want, tol)
    out = strided(torch.zeros(T, H), 5, 1).to(dt) if dt != F32 else strided(torch.zeros(T, H), 5, 1)
    assert few(x.cuda(), r, out=out) is out and torch.equal(out, y)  # and again: the same bits
    few.check()


def small_layer(fmt="nvfp4", E=4, H=192, I=96, seed=7):
    rng = gen(seed)
    up, _, _, _ = make_linear(rng, (E, 2 * I, H), fmt, False)
    down, _, _, _ = make_linear(rng, (E, H, I), fmt, False)
    up.tensor_scale.mul_(2.0 ** -10)
    down.tensor_scale.mul_(2.0 ** -10)
    return fp4.FewTokens(up, down)


@pytest.mark.parametrize("fmt", FORMATS)
def test_layer_rows_that_are_left_out(fmt):
    few = small_layer(fmt)
    x = torch.randn(6, 192, device="cuda")
    ids = np.array([[0, 1], [-1, -1], [2, -1], [3, 3], [-1, 0], [1, 2]])
    w = np.ones((6, 2), dtype=np.float32)
    w[1], w[2, 1] = np.nan, np.nan  # of choices that are none
    x[1] = float("nan")
    y = few(x, routing_of(ids, 4, w))
    assert torch.isfinite(y).all() and not y[1].any() and y[[0, 2, 3, 4, 5]].any(1).all()
    nothing = few(x, routing_of(np.full((6, 2), -1), 4))
    assert not nothing.any()
    assert few(x[:0], routing_of(np.zeros((0, 2), dtype=np.int64), 4)).shape == (0, 192)
    # an infinity or a NaN makes its own token NaN, nobody else
    x = torch.randn(6, 192, device="cuda")
    clean = few(x, routing_of(ids, 4))
    x[0, 3], x[5, 191] = float("inf"), float("nan")
    y = few(x, routing_of(ids, 4))
    assert y[[0, 5]].isnan().all() and torch.equal(y[1:5], clean[1:5])


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e25])
def test_layer_of_small_and_large_inputs(size):
    """relu without a gate is homogeneous: the input's size comes out as it went in (in 32 bits)."""
    rng = gen(8)
    up, _, _, _ = make_linear(rng, (2, 64, 128), "nvfp4", False)
    down, _, _, _ = make_linear(rng, (2, 128, 64), "nvfp4", False)
    few = fp4.FewTokens(up, down, "relu", gated=False)
    x = torch.from_numpy(rng.standard_normal((3, 128)).astype(np.float32)).cuda()
    r = routing_of(some_ids(rng, 3, 2, 2), 2)
    scale = float(2.0 ** np.round(np.log2(size)))
    assert torch.equal(few(x * scale, r) / scale, few(x, r))


def test_layer_in_place_with_an_expert_twice_and_rows_that_begin_later():
    few = small_layer()
    x = torch.randn(3, 192, device="cuda")
    once, twice = few(x, routing_of(np.array([[2], [0], [1]]), 4)), few(x, routing_of(np.array([[2, 2], [0, 0], [1, 1]]), 4))
    assert torch.equal(once + once, twice)
    # offsets may begin after 0: rows in front of them belong to nobody
    r = routing_of(np.array([[2], [0], [1]]), 4)
    late = ex.Routing(r.ids, r.weights, r.counts, r.offsets + 0, r.slots, r.source)
    late.offsets[0] = 1  # the row of expert 0, token 1's
    y = few(x, late)
    assert torch.equal(y[[0, 2]], once[[0, 2]]) and not y[1].any()
    z = x.clone()
    assert few(z, routing_of(np.array([[2], [0], [1]]), 4), out=z) is z and torch.equal(z, once)


@pytest.mark.parametrize("lo,hi", [(63, 64), (20, 23), (0, 2)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_layer_of_a_share_of_a_larger_routing(fmt, lo, hi):
    """Some of the experts, with the offsets of all choices' rows: the same bits as those choices alone, the others being none. Many parts of K, and far more rows than the share has."""
    rng = gen(14)
    T, k, E, H, I = 64, 32, 64, 4100, 40
    ids = some_ids(rng, T, k, E)
    w = rng.standard_normal((T, k)).astype(np.float32)
    up, _, _, _ = make_linear(rng, (hi - lo, 2 * I, H), fmt, False)
    down, _, _, _ = make_linear(rng, (hi - lo, H, I), fmt, False)
    up.tensor_scale.mul_(2.0 ** -10)
    few = fp4.FewTokens(up, down)
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32)).cuda()
    r = routing_of(ids, E, w)
    share = ex.Routing(r.ids, r.weights, r.counts[lo:hi].clone(), r.offsets[lo:hi + 1].clone(), r.slots, r.source)
    alone = routing_of(np.where((ids >= lo) & (ids < hi), ids - lo, -1), hi - lo, w)
    y = few(x, share)
    assert y.any() and torch.equal(y, few(x, alone))
    few.check()


def test_layer_refusals():
    few = small_layer()
    rng = gen(9)
    r = routing_of(some_ids(rng, 3, 2, 4), 4)
    x = torch.zeros(3, 192, device="cuda")
    refused(hb.ERR_COUNT_MISMATCH, lambda: few(x[:, :191], r))
    refused(hb.ERR_COUNT_MISMATCH, lambda: few(x[:2], r))
    refused(hb.ERR_COUNT_MISMATCH, lambda: few(x, routing_of(some_ids(rng, 3, 2, 5), 5)))
    refused(hb.ERR_DTYPE, lambda: few(x.double(), r))
    refused(hb.ERR_DTYPE, lambda: few(x, r, out=torch.zeros(3, 192, device="cuda", dtype=BF16)))
    refused(hb.ERR_INVALID_ARG, lambda: few(x.clone().requires_grad_(), r))
    refused(hb.ERR_INVALID_ARG, lambda: few(torch.zeros(65, 192, device="cuda"), routing_of(some_ids(rng, 65, 2, 4), 4)))
    refused(hb.ERR_INVALID_ARG, lambda: fp4.FewTokens(few.up, few.down, "tanh"))
    refused(hb.ERR_COUNT_MISMATCH, lambda: fp4.FewTokens(few.up, few.down, gated=False))
    refused(hb.ERR_COUNT_MISMATCH, lambda: fp4.FewTokens(few.down, few.up))
    refused(hb.ERR_DTYPE, lambda: fp4.FewTokens(few.up, small_layer("mxfp4").down))
    one = fp4.Fp4Linear(torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 4), dtype=torch.uint8, device="cuda"))
    refused(hb.ERR_INVALID_ARG, lambda: fp4.FewTokens(one, one))


# ------------------------------------------------------------------------------------------------ together, and as they are used
def test_a_run_of_them_together():
    """Route, the layer for few tokens; and the same tokens by rows in 4 bits, both products, activation and combine: apart by what rounding rows to 4 bits costs."""
    from paper_2608_00358_b200.activation import activate
    g = torch.Generator(device="cuda").manual_seed(1)
    E, k, H, I, T = 16, 4, 512, 256, 24
    w_up, w_down = (torch.randn(s, device="cuda", generator=g) * s[-1] ** -0.5 for s in ((E, 2 * I, H), (E, H, I)))
    x, logits = torch.randn(T, H, device="cuda", generator=g), torch.randn(T, E, device="cuda", generator=g)
    for fmt in FORMATS:
        up, down = (fp4.Fp4Linear.from_float(w, format=fmt) for w in (w_up, w_down))
        four = ref.rounded(np.array([[4.0]]), fmt)[0, 0]
        r = ex.Router(E, k).route(logits)
        y = fp4.FewTokens(up, down)(x, r)
        rows = fp4.quantize_rows(x, fmt, routing=r)
        h = activate(up.matmul(rows, offsets=r.offsets, dtype=F32), offsets=r.offsets)
        z = ex.combine(down(h, offsets=r.offsets), r)
        assert torch.equal(up.matmul(rows, offsets=r.offsets, dtype=F32), up(x, routing=r))
        # two roundings to 4 bits, each of about a tenth of a row's size, against none
        assert 0.01 < float((y - z).norm() / z.norm()) < 0.4
        exact = torch.zeros_like(x, dtype=torch.float64)
        for e in range(E):
            we = [(lin(torch.eye(n, device="cuda") * 4, offsets=torch.where(torch.arange(E + 1, device="cuda") > e, n, 0).int()) / four).double() for lin, n in ((up, H), (down, I))]
            u = x.double() @ we[0]
            exact += ((r.ids == e) * r.weights.double()).sum(1)[:, None] * ((torch.nn.functional.silu(u[:, :I]) * u[:, I:]) @ we[1])
        assert float((y - exact).norm() / exact.norm()) < 1e-5


def test_captured_and_replayed_on_other_streams():
    few, rng = small_layer(), gen(10)
    lin, _, _, _ = make_linear(rng, (256, 192), "nvfp4", False)
    r = routing_of(some_ids(rng, 5, 2, 4), 4)
    x = torch.randn(5, 192, device="cuda")
    big = torch.randn(300, 192, device="cuda")
    want = few(x, r), lin(big), lin(x)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = few(x, r), lin(big), lin(x)
        graphs.append((g, out))
    x2, big2 = torch.randn_like(x), torch.randn_like(big)
    want2 = few(x2, r), lin(big2), lin(x2)
    for inputs, expected in (((x2, big2), want2), ((x.clone(), big.clone()), want)):
        x.copy_(inputs[0])
        big.copy_(inputs[1])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in graphs]
        for _ in range(3):  # both graphs at once, and eager calls beside them
            for s, (g, _) in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
            few(x, r)
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, expected))
    few.check()
    lin.check()


def test_streams_and_threads_do_not_share_scratch():
    few = small_layer(H=1024, I=512)
    rng = gen(11)
    xs = [torch.randn(8, 1024, device="cuda") for _ in range(4)]
    rs = [routing_of(some_ids(rng, 8, 2, 4), 4) for _ in range(4)]
    want = [few(x, r) for x, r in zip(xs, rs)]
    bad = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream() if i % 2 else torch.cuda.default_stream()):
                for _ in range(50):
                    y = few(xs[i], rs[i])
                torch.cuda.current_stream().synchronize()
                if not torch.equal(y, want[i]):
                    bad.append(i)
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_writes_through_out_are_seen():
    few = small_layer()
    r = routing_of(np.array([[0, 1]]), 4)
    out = torch.zeros(1, 192, device="cuda")
    v = out._version
    few(torch.zeros(1, 192, device="cuda"), r, out=out)
    assert out._version > v
    refused(hb.ERR_INVALID_ARG, lambda: few(torch.zeros(1, 192, device="cuda"), r, out=out.requires_grad_()))


@pytest.mark.parametrize("seed", range(12))
def test_random_products_and_layers(seed):
    rng = gen(100 + seed)
    fmt, dt = FORMATS[seed % 2], (F32, BF16, F16)[seed % 3]
    M, N, K = int(rng.integers(1, 700)), int(rng.integers(1, 700)), int(rng.integers(1, 1500))
    lin, w, wide, b = make_linear(rng, (N, K), fmt, seed % 4 == 0)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(dt)
    within(lin(x.cuda()), *product(ref.rounded(x.float().numpy(), fmt), w[0], wide[0], None if b is None else b[0], dt))
    T, H, I, E = int(rng.integers(1, 30)), int(rng.integers(1, 600)), int(rng.integers(1, 400)), int(rng.integers(1, 9))
    k = int(rng.integers(1, E + 1))
    up, wu, gu, bu = make_linear(rng, (E, 2 * I, H), fmt, False)
    down, wd, gd, bd = make_linear(rng, (E, H, I), fmt, False)
    for lin, n in ((up, H), (down, I)):
        lin.tensor_scale.mul_(1 / (np.sqrt(n) * 150 if fmt == "nvfp4" else np.sqrt(n) / 4))
    gu, gd = up.tensor_scale.double().cpu().numpy(), down.tensor_scale.double().cpu().numpy()
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32)).to(dt)
    ids = some_ids(rng, T, k, E, 0.1)
    wt = rng.random((T, k)).astype(np.float32)
    want, tol = layer_reference(x.double().numpy(), ids, wt.astype(np.float64), (wu, gu, bu), (wd, gd, bd), "silu", True, fmt, dt)
    within(fp4.FewTokens(up, down)(x.cuda(), routing_of(ids, E, wt)), want, tol)
