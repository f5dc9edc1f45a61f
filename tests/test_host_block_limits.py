"""Limits that include/xattn.h states, on the host (no GPU needed): a scale inside them gets as far as the check of the workspace."""
import ctypes

import pytest

from paper_2512_16093_amd import binding as sla

FAKE = ctypes.c_void_p(0x1000)      # non-NULL, 16-byte aligned, never dereferenced


@pytest.mark.parametrize("scale,status", [(0.0, sla.ERR_WORKSPACE), (1e-30, sla.ERR_WORKSPACE), (1.0, sla.ERR_WORKSPACE),
                                          (1e30, sla.ERR_WORKSPACE), (0.99e-30, sla.ERR_VALUE), (1.01e30, sla.ERR_VALUE),
                                          (5e-324, sla.ERR_VALUE), (1e300, sla.ERR_VALUE)])
def test_range_of_the_scale_of_cross_attention(scale, status):
    L = sla.lib()
    assert L.xattn_fwd(FAKE, FAKE, FAKE, FAKE, None, None, None, None, None, None, 1, 2, 2, 5, 7, 128, scale, None, 0, None) == status
    assert L.xattn_bwd(*[FAKE] * 9, None, None, 1, 2, 2, 5, 7, 128, scale, None, 0, None) == status
