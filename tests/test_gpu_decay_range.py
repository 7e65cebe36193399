"""The decay mixer at the ends of the documented ranges: sums that are finite come out finite."""
import math

import pytest
import torch

from paper_2508_12594_amd import binding
from tests import _plain
from tests.test_gpu_decay import back, check, magnitudes, make

pytestmark = pytest.mark.gpu


def run(dev, wide, scale, dtype, N, d):
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    o, s = binding.decay_forward(*args, scale, want_state=True)
    *grads, ds = binding.decay_backward(*args, dev["d_o"], scale, want_dstate=True)
    names = ("q", "k", "v", "log_decay")
    want, size = (_plain.decay(*(w[n] for n in names), scale) for w in (wide, magnitudes(wide)))
    wgrad, gsize = (_plain.decay_gradients(*(w[n] for n in names), w["d_o"], scale) for w in (wide, magnitudes(wide)))
    fine = dtype if dtype == "f16" else "f32"
    for name, got, exact, mag in zip(("o", "dq", "dk", "dv", "state", "dstate"), [o] + grads + [s, ds],
                                     want[:1] + wgrad[:3] + (want[1], wgrad[3]), size[:1] + gsize[:3] + (size[1], gsize[3])):
        states = name in ("state", "dstate")
        check(name, back(got, "bhnd"), exact, mag, fine if states else dtype, N, d, 1 if states else 2)


@pytest.mark.parametrize("large_first", [False, True])
def test_fp16_small_terms_behind_a_large_sum(large_first):
    """Products of 2^32 at one end, fading subnormals before them: the common power of two that lifts these must not lift the sum past
    the end of fp32."""
    N, d = 1024, 32
    print("[case] fp16, large %s" % ("first" if large_first else "last"), flush=True)
    dev, wide = make(1, 2, N, d, "f16", 3, decays=[-2.0 * math.log(2.0), -2.0 * math.log(2.0)])
    tiny, large = 2.0 ** -24, 65000.0
    end = slice(0, 32) if large_first else slice(N - 32, N)
    for n in ("q", "k", "v", "d_o"):
        dev[n].fill_(tiny)
    for n in ("q", "d_o") if large_first else ("k", "v"):
        dev[n][:, :, end] = large
        dev[n][:, 1, :, ::2] *= -1
    for n in ("q", "k", "v", "d_o"):
        wide[n] = dev[n].double().cpu()
    run(dev, wide, 1.0, "f16", N, d)


@pytest.mark.parametrize("dtype,N", [("f32", 120), ("bf16", 300), ("bf16", 700)])
def test_large_states_of_wide_types(dtype, N):
    """Values of 1e31: what a slow decay leaves is kept as a factor beside the state, which must not leave fp32 for that.  (The first
    two sequences are not cut into segments.)"""
    d = 32
    decays = [-halvings * math.log(2.0) / 32 for halvings in (15.9, 9.0, 7.9, 3.0)]
    print("[case] 1e31 %s" % dtype, flush=True)
    dev, wide = make(1, 4, N, d, dtype, 7, decays=decays)
    dev["v"] = dev["v"] * 1e31
    wide["v"] = dev["v"].double().cpu()
    run(dev, wide, 0.1, dtype, N, d)
