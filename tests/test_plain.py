"""The plain 64-bit implementations that the GPU tests compare with, against torch's automatic derivatives and closed forms."""
import math

import pytest
import torch

from tests import _plain


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, dtype=torch.float64)


@pytest.mark.parametrize("lengths,carried", [(None, False), ([5, 0, 3], True)])
def test_decay_gradients_are_the_derivatives(lengths, carried):
    gen = torch.Generator().manual_seed(1)
    B, H, N, d = 3, 2, 5, 4
    q, k, v, d_o = (rand(gen, B, H, N, d) for _ in range(4))
    g = torch.tensor([-0.3, 0.0])
    state, ds = (rand(gen, B, H, d, d), rand(gen, B, H, d, d)) if carried else (None, None)
    lens = None if lengths is None else torch.tensor(lengths)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v) + ((state,) if carried else ())]
    o, s = _plain.decay(*leaves[:3], g, 0.7, lens, leaves[3] if carried else None)
    loss = (o * d_o).sum() + ((s * ds).sum() if carried else 0)
    want = torch.autograd.grad(loss, leaves)
    got = _plain.decay_gradients(q, k, v, g, d_o, 0.7, lens, state, ds)
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)


def test_decay_closed_form():
    """o_i = scale * (sum_j l^(i-j) <q_i,k_j> v_j + l^(i+1) state^T q_i)."""
    gen = torch.Generator().manual_seed(2)
    q, k, v, state = rand(gen, 1, 1, 6, 3), rand(gen, 1, 1, 6, 3), rand(gen, 1, 1, 6, 3), rand(gen, 1, 1, 3, 3)
    o, s = _plain.decay(q, k, v, torch.tensor([-0.4], dtype=torch.float64), 2.0, None, state)
    for i in range(6):
        want = math.exp(-0.4 * (i + 1)) * (q[0, 0, i] @ state[0, 0])
        for j in range(i + 1):
            want = want + math.exp(-0.4 * (i - j)) * (q[0, 0, i] @ k[0, 0, j]) * v[0, 0, j]
        assert torch.allclose(o[0, 0, i], 2.0 * want, rtol=1e-12)


@pytest.mark.parametrize("pre,post,gate_act,biases", [("layer", "rms", "silu", True), ("rms", "layer", "sigmoid", False),
                                                      ("none", "none", "none", False), ("layer", "none", None, True)])
def test_residual_norm_gradients_are_the_derivatives(pre, post, gate_act, biases):
    gen = torch.Generator().manual_seed(3)
    rows, C = 4, 7
    t = dict(x=rand(gen, rows, C), y=rand(gen, rows, C))
    if gate_act:
        t["gate"] = rand(gen, rows, C)
    for side, kind in (("pre", pre), ("post", post)):
        if kind != "none":
            t[side + "_weight"] = rand(gen, C)
            if biases:
                t[side + "_bias"] = rand(gen, C)
    leaves = {n: a.clone().requires_grad_(True) for n, a in t.items()}
    p = lambda s: {n: a for n, a in s.items() if "_" in n}   # noqa: E731
    x_out, h, _ = _plain.residual_norm(leaves["x"], leaves["y"], leaves.get("gate"), p(leaves), pre, post, gate_act, 0.6, 1e-5)
    dx_out, dh = rand(gen, rows, C), rand(gen, rows, C)
    loss = (x_out * dx_out).sum() + (0 if h is None else (h * dh).sum())
    want = dict(zip(leaves, torch.autograd.grad(loss, list(leaves.values()))))
    got = _plain.residual_norm_gradients(t["x"], t["y"], t.get("gate"), p(t), pre, post, gate_act, 0.6, 1e-5, dx_out,
                                         None if pre == "none" else dh)
    for n, w in want.items():
        assert torch.allclose(got[n], w, rtol=1e-10, atol=1e-12), n
