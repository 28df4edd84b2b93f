"""Operators in 4-bit floating point on the GPU, where the other tests do not reach: matrices' own scales in both formats."""
import copy
import pickle

import numpy as np
import pytest
import torch

import fp4_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import fp4
from test_gpu_experts import BF16, F16, F32, gen, strided
from test_gpu_fp4 import FORMATS, cuda, make_linear, product, refused, routing_of, some_ids, within

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
