"""Operators in 4-bit floating point on the GPU, where the other tests do not reach: matrices' own scales in both formats, scratch, large tiles one after the other, outliers, rows in 4 bits across
an exchange."""
import copy
import pickle

import numpy as np
import pytest
import torch

import expert_reference as eref
import fp4_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex
from paper_2608_00358_b200 import fp4
from paper_2608_00358_b200.activation import activate
from paper_2608_00358_b200.runtime import DeviceCollective
from test_gpu_experts import BF16, F16, F32, gen, strided
from test_gpu_fp4 import FORMATS, cuda, layer_reference, make_linear, product, refused, routing_of, some_ids, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("experts", [0, 3])
def test_a_matrixs_own_scale_counts_in_both_formats(experts, fmt):
    """A tensor_scale that is given is multiplied with, and copies of a layer have it too, whether it was given or changed in place."""
    rng = gen(21)
    N, K, G = 40, 96, max(experts, 1)
    flat, scale, values = ref.weights(rng, ((experts,) if experts else ()) + (N, K), fmt)
    wide = (0.5 + rng.random(G)).astype(np.float32)
    lin = fp4.Fp4Linear(cuda(flat), cuda(scale), cuda(wide), format=fmt)
    x = rng.standard_normal((6, K)).astype(np.float32)
    e = experts // 2
    off = torch.tensor([0] * (e + 1) + [6] * (experts - e), dtype=torch.int32, device="cuda") if experts else None
    want, tol = product(ref.rounded(x, fmt), values.reshape(G, N, K)[e], float(wide[e]), None, F32)
    y = lin(cuda(x), offsets=off)
    within(y, want, tol)
    lin.tensor_scale.mul_(0.5)  # a power of two: the same sums
    for f in (lambda v: v, copy.copy, copy.deepcopy, lambda v: pickle.loads(pickle.dumps(v))):
        assert torch.equal(f(lin)(cuda(x), offsets=off) * 2, y)
    refused(hb.ERR_COUNT_MISMATCH, lambda: fp4.Fp4Linear(cuda(flat), cuda(scale), torch.ones(G + 1, device="cuda"), format=fmt))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,H,I,E,k", [(1, 512, 256, 8, 8), (40, 264, 136, 3, 2), (64, 4100, 40, 32, 4), (3, 96, 2100, 2, 2)])
def test_scratch_may_hold_anything(monkeypatch, T, H, I, E, k, fmt):
    """The layer and the products give the same bits whatever earlier calls left in their scratch."""
    rng = gen(T)
    up, _, _, _ = make_linear(rng, (E, 2 * I, H), fmt, False)
    down, _, _, _ = make_linear(rng, (E, H, I), fmt, False)
    for lin in (up, down):
        lin.tensor_scale.mul_(2.0 ** -10)
    few = fp4.FewTokens(up, down)
    x = cuda(rng.standard_normal((T, H)).astype(np.float32))
    r = routing_of(some_ids(rng, T, k, E, 0.1), E)
    seen = []

    class Filled:
        def __init__(self, byte):
            self.byte = byte

        def get(self, dev, stream, nbytes):
            t = torch.full((nbytes,), self.byte, dtype=torch.uint8, device="cuda")
            seen.append(nbytes)
            return t, t.data_ptr()

    results = []
    for byte in (0, 0xFF, 0x7F, 0x3A):
        monkeypatch.setattr(fp4, "_scratch", Filled(byte))
        n = int(r.offsets[-1])
        results.append((few(x, r), up(x, routing=r)[:n], up.matmul(fp4.quantize_rows(x, fmt, routing=r), offsets=r.offsets)[:n]))
    assert len(seen) == 12 and results[0][0].any() and torch.isfinite(results[0][0]).all()
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    few.check()
    up.check()


# ------------------------------------------------------------------------------------------------ every tile, and several of them to a block
def tile_of(M, N, K, G, fmt):
    """The tokens of the tile that the library takes for a product, which its scratch's size tells."""
    stages, atoms = -(-K // 256), 4 if fmt == "nvfp4" else 2
    rows = -(-M * (-(-((K + 1) // 2) // 16) * 16) // 512) * 512
    have = hb.hccl_fp4_scratch_bytes(M, N, K, G, fp4.FORMATS[fmt])
    found = [tn for tn in (16, 32, 64, 128, 256) if rows + (-(-M // tn) + max(G, 1)) * max(tn // 128, 1) * stages * atoms * 512 == have]
    assert len(found) == 1, found
    return found[0]


def product_on_the_device(values, w, factor, bias, dt):
    """`product` of test_gpu_fp4 in 64 bits on the device: (y, tolerance)."""
    y, size = values @ w.t() * factor, values.abs() @ w.abs().t() * abs(factor)
    if bias is not None:
        y, size = y + bias, size + bias.abs()
    return y, (values.shape[1] + 4) * 2.0 ** -23 * size + eref.HALF_ULP[dt] * y.abs() * 1.01 + eref.SMALLEST[dt]


def inside(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K,dt,bias,tile", [
    (512, 4096, 4096, BF16, False, 128), (1500, 1410, 2050, F16, True, 128),   # one tile to a block
    (2000, 2600, 1100, F32, False, 128), (3333, 2222, 555, BF16, True, 128),   # 336 and 486 tiles over 148 blocks
    (520, 4200, 3000, BF16, False, 256),                                       # one to a pair
    (2700, 2701, 1300, F32, True, 256), (4499, 2900, 1290, BF16, False, 256), (2700, 2700, 1300, F16, False, 256),  # 121 and 216 over 74 pairs; 18 tiles of tokens
])
def test_large_tiles_one_after_the_other(M, N, K, dt, bias, tile, fmt):
    """Tiles of 128 and 256 tokens, several to a block or a pair: accumulators and stages used again, bands of eight tiles of tokens, ragged ends."""
    assert tile_of(M, N, K, 0, fmt) == tile
    rng = gen(M + N)
    lin, w, wide, b = make_linear(rng, (N, K), fmt, bias, 0.0173 if fmt == "nvfp4" else 1.0)
    if dt == F16:
        lin.tensor_scale.mul_(2.0 ** -10), wide.__imul__(2.0 ** -10)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(dt)
    values = cuda(ref.rounded(x.float().numpy(), fmt, lin.x_scale))
    want, tol = product_on_the_device(values, cuda(w[0]), float(wide[0]), None if b is None else cuda(b[0]), dt)
    y = lin(strided(x.cuda(), 3, 1))
    inside(y, want, tol)
    out = strided(torch.zeros(M, N), 7, 1).to(dt) if dt != F32 else strided(torch.zeros(M, N), 7, 1)  # no two results of a row side by side in one word
    lin(x.cuda(), out=out)
    assert torch.equal(out, y)
    assert torch.equal(lin.matmul(fp4.quantize_rows(x.cuda(), fmt, lin.x_scale), dtype=dt), y)
    lin.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,E,k,N,K,dt,tile", [(900, 60, 4, 700, 520, F32, 128), (1100, 70, 4, 1027, 320, BF16, 128), (3000, 3, 2, 1300, 700, F32, 256), (2500, 5, 4, 1030, 388, BF16, 256), (6000, 3, 2, 770, 264, F16, 256)])
def test_large_tiles_over_experts(T, E, k, N, K, dt, tile, fmt):
    """The same with rows of experts, which end anywhere in a tile: more than 148 tiles, or 74 for pairs, and an expert without rows."""
    rows = T * k
    assert tile_of(rows, N, K, E, fmt) == tile
    rng = gen(T + E)
    lin, w, wide, b = make_linear(rng, (E, N, K), fmt, T % 1000 == 0)
    if dt == F16:
        lin.tensor_scale.mul_(2.0 ** -10), wide.__imul__(2.0 ** -10)
    x = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).to(dt)
    ids = some_ids(rng, T, k, E, 0.1)
    ids[ids == E - 1] = 0
    r = routing_of(ids, E)
    offsets, n = r.offsets.tolist(), int(r.offsets[-1])
    assert sum(-(-(hi - lo) // tile) for lo, hi in zip(offsets, offsets[1:])) * -(-N // (256 if tile == 256 else 128)) > (74 if tile == 256 else 148)
    values = cuda(ref.rounded(x.float().numpy(), fmt))[(r.source.long() // k).clamp(min=0)]
    y = torch.full((rows, N), 77.0, dtype=dt, device="cuda")
    lin(x.cuda(), routing=r, out=y)
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:
            inside(y[lo:hi], *product_on_the_device(values[lo:hi], cuda(w[e]), float(wide[e]), None if b is None else cuda(b[e]), dt))
    assert (y[n:] == 77).all()
    z = torch.full((rows, N), 77.0, dtype=dt, device="cuda")
    lin.matmul(fp4.quantize_rows(x.cuda(), fmt, routing=r), offsets=r.offsets, out=z)
    assert torch.equal(y, z)
    lin.check()


# ------------------------------------------------------------------------------------------------ the layer beside outliers
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,H,I,E,k,size", [(5, 512, 256, 4, 2, 1e3), (33, 1100, 130, 3, 2, 1e4), (2, 2056, 1100, 4, 4, 4e5)])
def test_layer_beside_outliers(T, H, I, E, k, size, fmt):
    """A few columns far above the others: what is lost of every element is 2^-22 of the largest of up to 1024 neighbours, no more. Of the outliers' own products nothing is left
    where their weights are 0, and the others' then stand alone."""
    rng = gen(T + H)
    up, wu, gu, _ = make_linear(rng, (E, 2 * I, H), fmt, False)
    down, wd, gd, _ = make_linear(rng, (E, H, I), fmt, False)
    cols = rng.integers(0, H // 2, 3) * 2
    q = up.weight
    for c in cols[:2]:  # the outliers' weights: zero codes for two of them
        q[..., c // 2] &= 0xF0
        wu[..., c] = 0
    for lin, n in ((up, H), (down, I)):
        lin.tensor_scale.mul_(1 / (np.sqrt(n) * 150 if fmt == "nvfp4" else np.sqrt(n) / 4))
    gu, gd = up.tensor_scale.double().cpu().numpy(), down.tensor_scale.double().cpu().numpy()
    x = rng.standard_normal((T, H)).astype(np.float32)
    x[:, cols[:2]] *= np.float32(size)
    ids, weights = some_ids(rng, T, k, E), rng.random((T, k)).astype(np.float32)
    want, tol = layer_reference(x.astype(np.float64), ids, weights.astype(np.float64), (wu, gu, None), (wd, gd, None), "silu", True, fmt, F32)
    few = fp4.FewTokens(up, down)
    within(few(cuda(x), routing_of(ids, E, weights)), want, tol)
    few.check()


# ------------------------------------------------------------------------------------------------ across an exchange
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R,k,tokens,hidden,inner", [(2, 1, 5, 64, 96), (8, 3, 40, 250, 512), (16, 2, 9, 129, 40)])
def test_rows_cross_an_exchange_in_4_bits(R, k, tokens, hidden, inner, fmt):
    """One expert to a rank: codes and scales of a row side by side in a send buffer, written there by the C call, through the device-resident AllToAllv, into the product as they arrive; the
    activation, the second product, the way back. The rows, and the layer's result, as they are without an exchange, bit for bit."""
    rng = gen(R)
    up, _, _, _ = make_linear(rng, (R, 2 * inner, hidden), fmt, False)
    down, _, _, _ = make_linear(rng, (R, hidden, inner), fmt, False)
    up.tensor_scale.mul_(2.0 ** -10), down.tensor_scale.mul_(2.0 ** -10)

    def one(lin, e):
        return fp4.Fp4Linear(lin.weight[e:e + 1, :, : (lin.K + 1) // 2], lin._rows_scale[e:e + 1], lin.tensor_scale[e:e + 1], format=fmt, K=lin.K)

    width, blocks = (hidden + 1) // 2, -(-hidden // fp4.BLOCK[fmt])
    at = ex._pad16(width)
    row = at + ex._pad16(blocks)
    n_send, n_recv = tokens * k, tokens * R
    counts = torch.zeros((R, R), dtype=torch.int64, device="cuda")
    x = [torch.from_numpy(rng.standard_normal((tokens, hidden)).astype(np.float32)).to(BF16).cuda() for _ in range(R)]
    logits = [torch.from_numpy(rng.standard_normal((tokens, R)).astype(np.float32)).cuda() for _ in range(R)]
    send, recv = ([torch.zeros((n, row), dtype=torch.uint8, device="cuda") for _ in range(R)] for n in (n_send, n_recv))
    result, back = ([torch.zeros((n, hidden + hidden % 2), dtype=BF16, device="cuda") for _ in range(R)] for n in (n_recv, n_send))
    router, routings, stream = ex.Router(R, k), [], torch.cuda.current_stream()
    for s in range(R):
        r = router.route(logits[s])
        counts[s] = r.counts
        routings.append(r)
        hb.hccl_quantize_rows_fp4(x[s].data_ptr(), hidden, tokens, hidden, hb.BF16, fp4.FORMATS[fmt], 1.0, hb.C.byref(r.record), send[s].data_ptr(), row, send[s].data_ptr() + at, row,
                                  n_send, stream.cuda_stream)
        rows = fp4.quantize_rows(x[s], fmt, routing=r)
        assert torch.equal(send[s][:, :width], rows.q) and torch.equal(send[s][:, at: at + blocks], rows.scale)

    def exchange(counts, n_from, n_to, elems, a, b):
        plan = hb.hccl_plan_alltoallv_dynamic(R, [n_from] * R, [n_to] * R, hb.BF16, elems)
        plan.set_dynamic_metadata(counts.data_ptr())
        dc = DeviceCollective(plan)
        dc.set_buffers([t.data_ptr() for t in a], [t.data_ptr() for t in b], keep=(a, b, counts))
        dc.execute(stream)
        dc.check()

    exchange(counts, n_send, n_recv, row // 2, send, recv)
    for d in range(R):
        m = int(counts[:, d].sum())
        off = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        rows = fp4.Fp4Rows(recv[d][:, :width], recv[d][:, at: at + blocks], hidden, fmt)
        h = activate(one(up, d).matmul(rows, offsets=off), offsets=off)
        one(down, d)(h, offsets=off, out=result[d][:, :hidden])
    counts_back = counts.t().contiguous()
    exchange(counts_back, n_recv, n_send, hidden + hidden % 2, result, back)
    for s, r in enumerate(routings):
        want = ex.combine(down(activate(up(x[s], routing=r), offsets=r.offsets), offsets=r.offsets), r)
        assert want.any() and torch.equal(ex.combine(back[s][:, :hidden], r), want), s


# ------------------------------------------------------------------------------------------------ the longest rows
LONGEST = 131072


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K,dt", [(5, 40, LONGEST, BF16), (300, 130, LONGEST - 1, F32), (70, 129, LONGEST, F16)])
def test_product_of_the_longest_rows(M, N, K, dt, fmt):
    rng = gen(M)
    lin, w, wide, _ = make_linear(rng, (N, K), fmt, False)
    lin.tensor_scale.mul_(2.0 ** -12), wide.__imul__(2.0 ** -12)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(dt)
    codes, scale = ref.quantise(x.float().numpy(), fmt)
    rows = fp4.quantize_rows(x.cuda(), fmt)
    assert np.array_equal(rows.q.cpu().numpy(), ref.pack(codes)) and np.array_equal(rows.scale.cpu().numpy(), scale)
    want = torch.from_numpy(ref.values(codes, scale, fmt).astype(np.float32))
    assert torch.equal(rows.dequantize().cpu(), want)
    inside(lin(x.cuda()), *product_on_the_device(want.double().cuda(), cuda(w[0]), float(wide[0]), None, dt))
    refused(hb.ERR_INVALID_ARG, lambda: fp4.quantize_rows(torch.zeros(1, LONGEST + 1, device="cuda"), fmt))
    lin.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,H,I,E,k", [(2, LONGEST, 24, 2, 2), (3, 40, LONGEST, 2, 1)])
def test_layer_of_the_longest_rows(T, H, I, E, k, fmt):
    rng = gen(H)
    up, wu, _, _ = make_linear(rng, (E, 2 * I, H), fmt, False)
    down, wd, _, _ = make_linear(rng, (E, H, I), fmt, False)
    for lin, n in ((up, H), (down, I)):
        lin.tensor_scale.mul_(1 / (np.sqrt(n) * 150 if fmt == "nvfp4" else np.sqrt(n) / 4))
    gu, gd = up.tensor_scale.double().cpu().numpy(), down.tensor_scale.double().cpu().numpy()
    x, ids, weights = rng.standard_normal((T, H)).astype(np.float32), some_ids(rng, T, k, E), rng.random((T, k)).astype(np.float32)
    want, tol = layer_reference(x.astype(np.float64), ids, weights.astype(np.float64), (wu, gu, None), (wd, gd, None), "silu", True, fmt, F32)
    few = fp4.FewTokens(up, down)
    within(few(cuda(x), routing_of(ids, E, weights)), want, tol)
    few.check()
