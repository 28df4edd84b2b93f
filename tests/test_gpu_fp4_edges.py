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
