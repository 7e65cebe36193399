"""How often the decay mixer rounds: 16-bit outputs are as far from the 64-bit result as that result rounded once.

An output that is rounded once is off by a random part of half a step; any further rounding of its terms to the same type adds an
error of the same size, so that the norm of the error grows by sqrt(2).  Operands held in two numbers of the type are off by 2^-8
(bf16) or 2^-11 (fp16) of that, and fp32 sums of a few hundred terms by less: a tenth more than one rounding is allowed, which
leaves room for a further error of 0.46 of it."""
import pytest
import torch

from paper_2508_12594_amd import binding
from tests import _plain
from tests.test_gpu_decay import back, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,N,d,dtype,layout,lengths", [
    (1, 3, 300, 32, "bf16", "bhnd", None), (1, 2, 700, 128, "bf16", "bnhd", None), (2, 2, 333, 64, "f16", "bnhd", [333, 170]),
    (1, 2, 520, 128, "f16", "bhnd", None), (2, 4, 290, 16, "bf16", "bnhd", [100, 290]), (3, 1, 600, 64, "bf16", "bhnd", None)])
def test_outputs_are_rounded_once(B, H, N, d, dtype, layout, lengths):
    print("[case] rounding B%d H%d N%d d%d %s %s %s" % (B, H, N, d, dtype, layout, lengths), flush=True)
    dev, wide = make(B, H, N, d, dtype, 5 * N + d, layout, lengths, state=True)
    scale = d ** -0.5
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    keep = dict(lengths=dev["lengths"], state=dev["state"], layout=layout)
    o, _ = binding.decay_forward(*args, scale, **keep)
    grads = binding.decay_backward(*args, dev["d_o"], scale, dstate_out=dev["dstate_out"], **keep)[:3]
    names = ("q", "k", "v", "log_decay")
    want = _plain.decay(*(wide[n] for n in names), scale, wide["lengths"], wide["state"])[:1]
    want += _plain.decay_gradients(*(wide[n] for n in names), wide["d_o"], scale, wide["lengths"], wide["state"],
                                   wide["dstate_out"])[:3]
    for name, got, exact in zip(("o", "dq", "dk", "dv"), (o,) + grads, want):
        once = (exact.to(dev["q"].dtype).double() - exact).norm()
        off = (back(got, layout) - exact).norm() / once
        print("[case]    %s: %.3f of one rounding" % (name, off), flush=True)
        assert off <= 1.1, name
