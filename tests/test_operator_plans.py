"""How the residual norm's backward is cut, read from the workspace it asks for (no GPU needed)."""
import ctypes

import pytest

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.binding import NormShape


@pytest.mark.parametrize("rows,C,rows_per_gate", [(128, 128, 2), (4096, 128, 2), (4096, 64, 8), (900, 250, 3), (6000, 2000, 5)])
def test_gates_of_few_rows_get_workgroups(rows, C, rows_per_gate):
    """Rows that share a gate take a round of a workgroup of their own, however few they are: four rounds a workgroup, up to 768
    workgroups.  (Each workgroup has four rows of C sums in the workspace.)"""
    size = ctypes.c_size_t(0)
    shape = NormShape(rows, C, binding.FLARE_BF16, 0, 1, 0, 2, rows_per_gate)
    assert binding.load().flare_residual_norm_workspace_bytes(ctypes.byref(shape), ctypes.byref(size)) == 0
    workgroups = size.value // (16 * C)
    assert workgroups >= min(rows // rows_per_gate // 4, 768) * 0.75       # (whole units each)
