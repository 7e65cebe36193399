"""The decay mixer and the residual norm have first derivatives: a second one raises, rather than come out without their part."""
import pytest
import torch

from paper_2508_12594_amd.autograd import decay_mixer, residual_norm
from paper_2508_12594_amd.binding import FlareError
from tests.test_gpu_decay import make

pytestmark = pytest.mark.gpu


def mixed(dev):
    return lambda t: t + decay_mixer(t, dev["k"], dev["v"], dev["log_decay"], 0.2, state=dev["state"], want_state=True)[0]


def normed(dev):
    return lambda t: t + residual_norm(t, dev["k"], post="rms")[1]


@pytest.mark.parametrize("which", [mixed, normed])
def test_a_penalty_on_a_gradient_raises(which):
    print("[case] second derivative of", which.__name__, flush=True)
    dev, _ = make(1, 2, 40, 32, "f32", 61, state=True)
    f = which(dev)
    x = dev["q"].clone().requires_grad_(True)
    plain, = torch.autograd.grad(f(x), x, dev["d_o"])
    grad, = torch.autograd.grad(f(x), x, dev["d_o"], create_graph=True)
    assert torch.equal(grad, plain) and grad.requires_grad
    with pytest.raises(FlareError, match="no second derivative"):
        torch.autograd.grad((f(x) * grad).sum(), x)
    # ... nor by the gradient that came in
    d = dev["d_o"].clone().requires_grad_(True)
    grad, = torch.autograd.grad(f(x), x, d, create_graph=True)
    with pytest.raises(FlareError, match="no second derivative"):
        torch.autograd.grad(grad.sum(), d)
    x.grad = None
    f(x).backward(dev["d_o"], create_graph=True)      # asked for, but not used
    assert torch.equal(x.grad.detach(), plain)
    x.grad = None


def test_traced_forms():
    print("[case] second derivative, traced", flush=True)
    dev, _ = make(1, 2, 40, 32, "f32", 61)
    x = dev["q"].clone().requires_grad_(True)
    for f in (lambda t: decay_mixer(t, dev["k"], dev["v"], dev["log_decay"], 0.2)[0], lambda t: residual_norm(t, dev["k"])[1]):
        traced = torch.jit.trace(f, (dev["k"],), check_trace=False)
        grad, = torch.autograd.grad(traced(x), x, dev["d_o"], create_graph=True)
        with pytest.raises(RuntimeError, match="no second derivative"):
            torch.autograd.grad((x * grad).sum(), x)
