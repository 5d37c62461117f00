"""More of what the 4-bit cache's entry points turn into a status or an error on the host (nothing below reaches a launch)."""
import pytest

from test_kv_refusals import HYPER, NULL, attend, batch, desc, strides


@pytest.mark.parametrize("scale,code", [(2.0 ** 100, NULL), (1.3e30, HYPER), (3.0e38, HYPER), (1e-45, NULL)])
def test_scales(scale, code):
    """up to 2^100 (the call without a pool goes on to its next refusal)"""
    assert attend(desc(), batch(), qs=strides(), os_=strides(), scale=scale, pool=None) == code
