"""CPU tests of the reader's calls beside the refusals of test_reader_abi.py."""
import ctypes

import pytest

from paper_2107_06960_amd import mafat as M
from paper_2107_06960_amd import operators as O
from test_reader_abi import CROSS


@pytest.mark.parametrize("scale, status", [(2.35e38, 0), (-2.35e38, 0), (2.37e38, M.MAFAT_EUNSUPPORTED),
                                           (-3.4e38, M.MAFAT_EUNSUPPORTED)])
def test_a_scale_has_to_be_finite_in_base_2(scale, status):
    n = ctypes.c_size_t()
    assert O.lib().mafat_cross_workspace(ctypes.byref(O.mafat_cross(**dict(CROSS, scale=scale))), ctypes.byref(n)) == status
