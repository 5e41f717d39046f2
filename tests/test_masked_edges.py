"""Arguments of masked attention at the ends of their ranges (no GPU needed)."""
import pytest
import torch

from paper_2401_11202_amd import partir as P
from tests.test_stream_checks import status


@pytest.mark.parametrize("kw", [dict(cap=1e-50), dict(cap=-1e-50), dict(scale=1e-50), dict(scale=2.0 ** -151)])
def test_numbers_that_float32_rounds_to_zero_do_not_select_what_zero_does(kw):
    x, lse = torch.zeros(4, 256, dtype=torch.bfloat16), torch.zeros(4, 2)
    sizes = dict(B=1, Sq=4, Sk=4, n_heads=2, **kw)
    for call in (lambda: P.masked_attention(x, x, x, **sizes), lambda: P.masked_attention_train(x, x, x, **sizes),
                 lambda: P.masked_attention_backward(x, x, x, x, x, lse, **sizes)):
        assert status(call) == "PARTIR_E_UNSUPPORTED"


@pytest.mark.parametrize("scale", [0.0, -0.0, -1e-50, -3.0])
def test_a_scale_that_is_not_positive_selects_the_default(scale):
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    assert status(lambda: P.masked_attention(x, x, x, B=1, Sq=4, Sk=4, n_heads=2, scale=scale)) == "PARTIR_E_LAYOUT"   # on the CPU
