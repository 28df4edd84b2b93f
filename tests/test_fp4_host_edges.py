"""Operators in 4-bit floating point, host side: what the Python layer says and does before a launch, on the CPU."""
import pytest
import torch

from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex
from paper_2608_00358_b200 import fp4


def test_refused_gradients_are_named_by_the_call_that_has_none():
    x = torch.zeros(2, 32, requires_grad=True)
    lin, few = object.__new__(fp4.Fp4Linear), object.__new__(fp4.FewTokens)
    lin.dev = few.dev = 0
    routing = type("R", (), dict(tokens=2, top_k=1, weights=torch.ones(2, 1, requires_grad=True)))()
    for call, says in ((lambda: fp4.quantize_rows(x), "x requires a gradient, and 4-bit rows have none"), (lambda: lin(x), "x requires a gradient, and 4-bit rows have none"),
                       (lambda: few(x, routing), "x requires a gradient, and FewTokens has none"),
                       (lambda: few(x.detach(), routing), "the routing's weights requires a gradient, and FewTokens has none"),
                       (lambda: ex.quantize_rows(x), "x requires a gradient, and 8-bit rows have none")):
        with pytest.raises(hb.HcclError) as e:
            call()
        assert e.value.status == hb.ERR_INVALID_ARG and says in str(e.value)
