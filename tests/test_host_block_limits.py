"""Limits that include/xattn.h states, and how cross attention deals out its work, on the host (no GPU needed).  A scale inside its
limits gets as far as the check of the workspace."""
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


@pytest.mark.parametrize("H,Nq,Nk,split", [
    (12, 2048, 2048, False),     # us in one piece and in two: 41.2, 51.9
    (40, 512, 2048, False),      # 41.2, 49.0
    (12, 4096, 4096, False),     # 113, 128
    (12, 2048, 1024, False),     # 23.3, 37.6
    (12, 1024, 512, False),      # 13.4, 21.8
    (12, 32760, 512, False),
    (12, 1024, 4096, True),      # 75.3, and in five 46.2
    (12, 2048, 8192, True),      # 148, in four 126
    (12, 256, 4096, True),       # 73.9, in eight 25.7
    (24, 300, 1500, True),       # 31.2, in three 26.6
    (12, 1, 512, True),          # 12.7, in eight 8.9
])
def test_walks_are_split_where_that_is_faster(H, Nq, Nk, split):
    """Cross attention's forward walk over the keys, on 256 compute units; a walk in one piece needs no workspace to speak of."""
    assert (sla.xattn_workspace_bytes(1, H, H, Nq, Nk, 128) > 256) == split
