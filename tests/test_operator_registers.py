"""What the compiler made of the decay mixer's and the residual norm's kernels, read from the metadata in the built library: the
counts of workgroups rest on these waves.  No GPU needed."""
import re

import pytest

from tests.test_kernel_registers import kernels  # noqa: F401

F32, BF16, F16 = 0, 1, 2


def found(kernels, pattern):   # noqa: F811
    out = {n: k for n, k in kernels.items() if re.search(pattern, n)}
    assert out, "no such kernels in the library"
    return out


@pytest.mark.parametrize("dtype,head,most", [(t, d, 256) for t in (BF16, F16) for d in (16, 32, 64, 128)] + [(F32, 16, 256), (F32, 32, 256),
                                             (F32, 64, 512), (F32, 128, 512)])
def test_scan_registers(kernels, dtype, head, most):   # noqa: F811
    """Two waves a SIMD (fp32 from d = 64 on: one), and nothing of the state in memory (fp16 at d = 128: two values a chunk)."""
    for n, k in found(kernels, r"decay_scan_kernelILi%dELi%dELi1E" % (dtype, head)).items():
        assert k[".vgpr_count"] <= most and k[".vgpr_spill_count"] <= (2 if (dtype, head) == (F16, 128) else 0), n
    if head < 128:
        for n, k in found(kernels, r"decay_scan_kernelILi%dELi%dELi2E" % (dtype, head)).items():
            assert k[".vgpr_count"] <= 256 and k[".vgpr_spill_count"] == 0, n
    for n, k in found(kernels, r"decay_sum_kernelILi%dELi%dE" % (dtype, head)).items():
        assert k[".vgpr_count"] <= 256 and k[".vgpr_spill_count"] == 0, n


def test_norm_registers(kernels):   # noqa: F811
    """No forward spills; of the backwards only those of 1024 lanes with a post norm or a gate, whose lanes have 128 registers, and
    a few values without."""
    for n, k in found(kernels, r"residual_norm_kernel").items():
        assert k[".vgpr_spill_count"] == 0, n
    for n, k in found(kernels, r"residual_norm_backward_kernel").items():
        if "Li1024E" not in n:
            assert k[".vgpr_spill_count"] == 0, n
        elif n.endswith("Lb0EEEvNS0_8NormArgsE"):
            assert k[".vgpr_spill_count"] <= 16, n
