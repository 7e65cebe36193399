"""Single tokens over a long run: the decay that is applied thousands of times is the exact one."""
import math

import pytest
import torch

from paper_2508_12594_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,B,by_step", [(32, 1, True), (128, 70, True), (64, 1, False)])
def test_steps_do_not_drift(d, B, by_step):
    """Tokens that add nothing (v = 0) leave l^T of the state.  Each step rounds each entry once, by at most u = 2^-24 and in no
    direction: T steps are beyond 8 sqrt(T) u with a probability of 2 exp(-32) (Hoeffding).  A factor that is rounded to 24 bits is off
    by up to u / 2 in every step the same way, T u / 2 in all: four times as much."""
    T, u = 4096, 2.0 ** -24
    reach = [512.0, 700.0, 1024.0, 1500.0, 3000.0, 5000.0, 8192.0, 16384.0]
    print("[case] long run d%d %s" % (d, "steps" if by_step else "sequences of one token"), flush=True)
    log_decay = torch.tensor([-1.0 / r for r in reach], device="cuda")
    H = len(reach)
    gen = torch.Generator(device="cuda").manual_seed(3)
    first = torch.randn(B, H, d, d, generator=gen, device="cuda")
    k = torch.randn(B, H, d, generator=gen, device="cuda")
    v = torch.zeros_like(k)
    state, o = first.clone(), torch.empty_like(k)
    for _ in range(T):
        if by_step:
            binding.decay_step(k, k, v, log_decay, state, 0.5, o=o)
        else:
            one = [t.unsqueeze(2) for t in (k, k, v, o)]
            binding.decay_forward(*one[:3], log_decay, 0.5, state=state, state_out=state, o=one[3])
    want = first.double() * (T * log_decay.double()).exp().view(1, H, 1, 1)
    off = ((state.double() - want).abs() / (want.abs() + 1e-30)).amax((0, 2, 3))
    print("[case]    off by (in u):", [round(x) for x in (off / u).tolist()], flush=True)
    assert (off <= 8 * math.sqrt(T) * u).all()
