"""What the calls write over is known to autograd: a backward pass that had saved it raises instead of using the new values."""
import pytest
import torch

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.autograd import decay_mixer, residual_norm
from tests.test_gpu_decay import make

pytestmark = pytest.mark.gpu


def test_a_state_in_place_behind_a_saved_one():
    print("[case] state in place", flush=True)
    dev, _ = make(2, 3, 50, 32, "bf16", 43, state=True)
    names = ("q", "k", "v", "log_decay")
    tok = [dev[n][:, :, 0].contiguous() for n in names[:3]]

    def overwritten(write):
        t = {n: dev[n].clone() for n in names + ("state",)}
        t["q"].requires_grad_(True)
        o, _ = decay_mixer(*(t[n] for n in names), 0.2, state=t["state"])
        write(t)
        return lambda: torch.autograd.grad(o, t["q"], dev["d_o"])

    for write in (lambda t: binding.decay_step(*tok, t["log_decay"], t["state"], 0.2),
                  lambda t: binding.decay_step(*tok, t["log_decay"], dev["state"], 0.2, state_out=t["state"]),
                  lambda t: binding.decay_forward(*(dev[n] for n in names), 0.2, state=t["state"], state_out=t["state"]),
                  lambda t: binding.decay_forward(*(dev[n] for n in names), 0.2, o=t["v"]),
                  lambda t: binding.decay_backward(*(dev[n] for n in names), dev["d_o"], 0.2, dk=t["k"]),
                  lambda t: binding.residual_norm_forward(dev["q"], dev["k"], x_out=t["v"])):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            overwritten(write)()
    fresh = torch.empty_like(dev["state"])
    untouched = overwritten(lambda t: binding.decay_step(*tok, t["log_decay"], t["state"], 0.2, state_out=fresh))()
    assert torch.equal(untouched[0], overwritten(lambda t: None)()[0])
    with torch.inference_mode():                    # tensors without versions
        state = torch.zeros_like(dev["state"])
        binding.decay_step(*tok, dev["log_decay"], state, 0.2, o=torch.empty_like(tok[0]))


def test_a_residual_stream_in_place():
    print("[case] residual stream in place", flush=True)
    x, y = torch.randn(2, 7, 64, device="cuda", requires_grad=True), torch.randn(2, 7, 64, device="cuda")
    _, h = residual_norm(x, y)
    binding.residual_norm_forward(x.detach(), y, x_out=x.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        h.sum().backward()
