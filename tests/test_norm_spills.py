"""Registers that the residual norm's backward of 1024 lanes keeps in memory: with a post norm or a gate its 128 a lane do not
suffice, and it is to get no worse.  Read from the built library's metadata; no GPU needed."""
import re

import pytest

from tests.test_kernel_registers import kernels  # noqa: F401


@pytest.mark.parametrize("whole,most", [(True, 96), (False, 168)])
def test_backward_of_1024_lanes(kernels, whole, most):   # noqa: F811
    """whole: C a multiple of eight (then the weights, too, come in 16-byte pieces)."""
    found = {n: k for n, k in kernels.items() if re.search("residual_norm_backward_kernelILi.ELi.ELi1024ELb%dELb1E" % whole, n)}
    assert len(found) == 5, "no such kernels in the library"
    for n, k in found.items():
        assert k[".vgpr_spill_count"] <= most, n
