"""CPU tests of the reader's calls beside the refusals of test_reader_abi.py."""
import ctypes
import glob
import os
import re

import pytest

from paper_2107_06960_amd import mafat as M
from paper_2107_06960_amd import operators as O
from test_reader_abi import CROSS, ROOT


def test_assembly_puts_m0_back():
    """The compiler may keep a value of its own in m0, and assembly cannot declare that register as overwritten."""
    found = 0
    for path in glob.glob(os.path.join(ROOT, "paper_2107_06960_amd", "csrc", "*")):
        for text in re.findall(r"\basm\s+volatile\s*\((.*?)\);", open(path).read(), re.S):
            if re.search(r"\bm0,", text):
                found += 1
                steps = [step.strip() for step in re.search(r'"(.*?)"\s*\n?\s*:', text, re.S).group(1).split(r"\n\t")]
                assert steps[0] == "s_mov_b32 %0, m0" and steps[-1] == "s_mov_b32 m0, %0", (path, steps)
    assert found


@pytest.mark.parametrize("scale, status", [(2.35e38, 0), (-2.35e38, 0), (2.37e38, M.MAFAT_EUNSUPPORTED),
                                           (-3.4e38, M.MAFAT_EUNSUPPORTED)])
def test_a_scale_has_to_be_finite_in_base_2(scale, status):
    n = ctypes.c_size_t()
    assert O.lib().mafat_cross_workspace(ctypes.byref(O.mafat_cross(**dict(CROSS, scale=scale))), ctypes.byref(n)) == status


def test_a_reader_without_adapters_refuses_the_rows_adapters():
    import torch
    from paper_2107_06960_amd import reader as R
    reader = R.Reader(R.draw_params(64, 2, 32, 1, device="cpu"), 2, 1, 32)
    with pytest.raises(ValueError, match="row_adapter"):
        reader.run(torch.zeros(2, 64), torch.zeros(1, 2, 2, 64), row_adapter=torch.zeros(2, dtype=torch.int32))
