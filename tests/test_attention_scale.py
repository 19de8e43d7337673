"""CPU-only: scales whose products with log2(e) are no fp32 numbers are refused by every call that takes a scale."""
import pytest

import paper_2602_05367_amd as rb
from test_attention_boundary import _grad, _paged, _prompt


@pytest.mark.parametrize("scale", [2.01e38, 2.4e38, 3e38, 3.4e38])
def test_scales_beyond_the_arithmetic(scale):
    assert _prompt(scale=scale) == rb.RB_ERR_VALUE and _grad(scale=scale) == rb.RB_ERR_VALUE and _paged(scale=scale) == rb.RB_ERR_VALUE
