"""Scales that binary32 cannot take times log2 e are refused (no GPU needed)."""
import pytest

from test_logprob_operators_host import bwd, fwd


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("scale", [3.4e38, 2.4e38, 1.8e38])
def test_scales_beyond_2_to_127(call, scale):
    assert call(scale=scale) == -6
