"""The slope of a sigmoid gate far out: sigmoid (1 - sigmoid) to the last bits, though the second factor is next to nothing."""
import pytest
import torch

from paper_2508_12594_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,sign", [(64, 1.0), (250, 1.0), (8192, 1.0), (64, -1.0)])
def test_slopes_of_wide_open_gates(C, sign):
    """exp(-g) is good to 2^-24 of its exponent's argument and a few steps (v_exp_f32, v_rcp_f32: 2^-23 each), the products to
    2^-24 each: 2 |g| + 16 units of 2^-24 in all."""
    print("[case] open gates C%d %+g" % (C, sign), flush=True)
    gen = torch.Generator().manual_seed(9)
    shape = (12, C)
    g = sign * (1 + 79 * torch.rand(shape, generator=gen))
    x, y, dx_out = (torch.randn(shape, generator=gen) for _ in range(3))
    grads = binding.residual_norm_backward(x.cuda(), y.cuda(), dx_out.cuda(), None, None, gate=g.cuda(), pre="none", gate_act="sigmoid",
                                           alpha=0.5)
    wide = g.double()
    want = 0.5 * dx_out.double() * y.double() * torch.exp(-wide) / (1 + torch.exp(-wide)) ** 2
    worst = ((grads[2].double().cpu() - want).abs() / want.abs() / ((2 * g.abs() + 16) * 2.0 ** -24)).max().item()
    print("[case]    worst error / tolerance %.3f" % worst, flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
def test_closed_gates(act):
    """A gate at its type's lowest value lets nothing through, in either direction."""
    print("[case] closed gates " + act, flush=True)
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        x, y, d = (torch.randn(5, 128, device="cuda").to(dt) for _ in range(3))
        g = torch.full_like(x, torch.finfo(dt).min)
        x_out, _ = binding.residual_norm_forward(x, y, g, pre="none", gate_act=act)
        dx, dy, dgate, *_ = binding.residual_norm_backward(x, y, d, None, None, gate=g, pre="none", gate_act=act)
        assert torch.equal(x_out, x) and torch.equal(dx, d) and (dy == 0).all() and (dgate == 0).all()
