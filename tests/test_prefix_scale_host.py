"""Scales that the group attention cannot take into base 2, refused before anything is launched.  No GPU."""
import ctypes as C

import pytest

from paper_2606_18967_amd import sdrl
from test_prefix_host import INVAL, PTR, cache


@pytest.mark.parametrize("scale", [2.5e38, -2.5e38, 3.4028234e38])
def test_a_scale_without_a_finite_base_2_scale_is_refused(scale):
    L, c = sdrl.lib(), cache()
    need = L.sd_prefix_workspace_bytes(C.byref(c), 1, 1, 4)
    assert L.sd_prefix_attention(C.byref(c), None, 0, 1, 1, PTR, None, 4, PTR, 512, scale, PTR, 512, PTR + 16, need, None) == INVAL
    assert b"scale" in L.sd_last_error()
