"""Options of the AdamW step that are finite in 64 bits and not in the 32 that the step works in are refused."""
import pytest
import torch

import paper_2512_11280_b200 as adasd
from tests.test_adamw_cpu import call


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the call goes on to look at the context, and there is none here")
@pytest.mark.parametrize("name", ["lr", "eps", "grad_scale"])
def test_options_beyond_32_bits(name):
    for sign in (1.0, -1.0):
        assert call(**{name: sign * 1e39}) == adasd.ERR_SHAPE
    assert call(**{name: 3e38}) not in (adasd.ERR_SHAPE, 0)
