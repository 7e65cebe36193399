"""Buffers that may not be one, refused on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.binding import NormShape

ONE = ctypes.c_float(1)
X, Y, O, H = (ctypes.c_void_p(i << 24) for i in range(1, 5))      # never dereferenced, and far from each other


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_an_fp32_stream_does_not_fit_16_bit_buffers(lib):
    """Beside 16-bit branches the rows of an fp32 residual stream are twice as long: neither may lie in the other's buffer."""
    shape = ctypes.byref(NormShape(10, 64, binding.FLARE_BF16, 1, 1, 0, 0, 1))
    fwd = lib.flare_residual_norm_forward
    assert fwd(shape, None, X, Y, None, Y, H, None, ONE, ONE, None) == -1          # x_out over y
    assert fwd(shape, None, X, Y, None, O, X, None, ONE, ONE, None) == -1          # h over x
    assert fwd(shape, None, X, None, None, None, X, None, ONE, ONE, None) == -1
