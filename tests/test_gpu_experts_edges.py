"""Expert-layer operators where it is easy to go wrong: rows with nothing left, groups by sums of scores, scores at the ends of their range, many experts in
many groups, gradients of every layout, autograd's own rules, host threads, and the sizes at which another kernel or another turn of a loop takes over."""
import numpy as np
import pytest
import torch

import expert_reference as ref
from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex
from test_gpu_experts import BF16, F16, F32, check_routing, cuda, gen, grid_logits, strided, weight_tol

pytestmark = pytest.mark.gpu


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
