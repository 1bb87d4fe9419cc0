"""Scales of attention scores that the calls refuse (no GPU needed)."""
import numpy as np
import pytest

from tests.test_attn_api import RANGE, cache, prompt


@pytest.mark.parametrize("call", [cache, prompt])
@pytest.mark.parametrize("scale", [2.4e38, 3.4e38, float(np.finfo(np.float32).max)])
def test_scales_whose_base_2_form_is_infinite_are_refused(call, scale):
    """The kernels count scores in powers of two: scale * log2(e) has to be finite in fp32, or scores of 0 are no numbers."""
    assert call(scale=scale) == RANGE


@pytest.mark.parametrize("call", [cache, prompt])
def test_the_largest_scales_pass(call):
    assert call(scale=2.3e38, **({"tokens": 0} if call is cache else {"tokens_q": 0})) == 0
