"""The decay mixer, the residual norm and the framework's own mixer together, as a model has them: training against 64-bit
automatic derivatives of the plain formulas, and generation (a padded batch of prompts, then single tokens) against one
long pass."""
import pytest
import torch

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.autograd import decay_mixer, flare_mixer, residual_norm
from tests import _plain

pytestmark = pytest.mark.gpu

B, N, H, D, M = 3, 70, 4, 16, 8
C = H * D
SCALE = D ** -0.5


def parameters(seed):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen)   # noqa: E731
    p = {"w%d" % i: rand(C, C) / C ** 0.5 for i in range(8)}
    p.update({"norm%d" % i: 1 + 0.1 * rand(C) for i in range(5)})
    p.update({"bias%d" % i: 0.1 * rand(C) for i in range(2)})
    p["layer_scale"] = 0.5 + 0.1 * rand(C)
    p["latents"] = rand(H, M, D)
    return p


DECAYS = [-1.0 / (4.0 * 2.0 ** h) for h in range(H)]


def heads(t):
    return t.view(t.shape[0], t.shape[1], H, D)


def model(p, x, lengths=None):
    """A causal block (decay mixer, gated, normed on both sides of the addition) and one of the framework's own blocks."""
    g = torch.tensor(DECAYS, device=x.device)
    _, h = residual_norm(x, pre_weight=p["norm0"], pre_bias=p["bias0"])
    o, _ = decay_mixer(heads(h @ p["w0"]), heads(h @ p["w1"]), heads(h @ p["w2"]), g, SCALE, lengths=lengths, layout="bnhd")
    x, h = residual_norm(x, o.reshape(x.shape) @ p["w3"], h @ p["w4"], pre="layer", post="rms", pre_weight=p["norm1"],
                         pre_bias=p["bias1"], post_weight=p["norm2"], gate_act="silu", alpha=0.7)
    y = flare_mixer(p["latents"], heads(h @ p["w5"]), heads(h @ p["w6"]), SCALE, layout="bnhd")
    x, h = residual_norm(x, y.reshape(x.shape) @ p["w7"], p["layer_scale"], pre="rms", post="rms", pre_weight=p["norm3"],
                         post_weight=p["norm4"])
    return x, h


def plain_model(p, x):
    def norm(t, kind, w=None, b=None):
        return _plain._one_norm(t.reshape(-1, C), kind, w, b, 1e-5)[2].reshape(t.shape)

    split = lambda t: heads(t).transpose(1, 2)   # noqa: E731
    merge = lambda t: t.transpose(1, 2).reshape(t.shape[0], t.shape[2], C)   # noqa: E731
    h = norm(x, "layer", p["norm0"], p["bias0"])
    o, _ = _plain.decay(split(h @ p["w0"]), split(h @ p["w1"]), split(h @ p["w2"]), torch.tensor(DECAYS).double(), SCALE)
    gate = h @ p["w4"]
    x = x + 0.7 * norm(merge(o) @ p["w3"], "rms", p["norm2"]) * gate * torch.sigmoid(gate)
    h = norm(x, "layer", p["norm1"], p["bias1"])
    k, v = split(h @ p["w5"]), split(h @ p["w6"])
    s = SCALE * torch.matmul(p["latents"], k.transpose(2, 3))
    y = torch.matmul(s.softmax(2).transpose(2, 3), torch.matmul(s.softmax(3), v))
    x = x + norm(merge(y) @ p["w7"], "rms", p["norm4"]) * p["layer_scale"]
    return x, norm(x, "rms", p["norm3"])


def test_a_training_step():
    """fp32: gradients of every parameter and of the input to 1e-4 of their size (a dozen operations of relative error below
    1e-6 each, the norms' scales between 1 and 3)."""
    print("[case] causal block, training", flush=True)
    gen = torch.Generator().manual_seed(2)
    x, dx, dh = (torch.randn(B, N, C, generator=gen) for _ in range(3))
    p = parameters(1)
    leaves = {n: t.cuda().requires_grad_(True) for n, t in dict(p, x=x).items()}
    out = model(leaves, leaves["x"])
    got = torch.autograd.grad(out, list(leaves.values()), [dx.cuda(), dh.cuda()])
    wide = {n: t.double().requires_grad_(True) for n, t in dict(p, x=x).items()}
    ref = plain_model(wide, wide["x"])
    want = torch.autograd.grad(ref, list(wide.values()), [dx.double(), dh.double()])
    for a, b in zip(out, ref):
        assert (a.double().cpu() - b).norm() <= 1e-5 * b.norm()
    for n, a, b in zip(leaves, got, want):
        error = ((a.double().cpu() - b).norm() / b.norm()).item()
        print("[case]    d%s %.1e" % (n, error), flush=True)
        assert error <= 1e-4, n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_then_single_tokens(dtype):
    """A padded batch of prompts through the causal block, its states kept, then tokens one by one: what one pass over the whole
    sequences gives.  (16 bits: every layer's output is rounded in both, 2^-8 a time: a few of these.)"""
    print("[case] causal block, generation %s" % dtype, flush=True)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(B, N, C, generator=gen).cuda().to(dt)
    p = {n: t.cuda() if n.startswith(("norm", "bias")) else t.cuda().to(dt) for n, t in parameters(3).items()}
    g = torch.tensor(DECAYS, device="cuda")
    lengths = [40, 1, 64]

    def before(t):
        _, h = binding.residual_norm_forward(t, pre_weight=p["norm0"], pre_bias=p["bias0"])
        return h, [heads(h @ p["w%d" % i]).contiguous() for i in range(3)]

    def after(t, o, h):
        return binding.residual_norm_forward(t, (o.reshape(t.shape) @ p["w3"]).contiguous(), (h @ p["w4"]).contiguous(), pre="rms",
                                             post="rms", pre_weight=p["norm1"], post_weight=p["norm2"], gate_act="silu")

    h, qkv = before(x)
    o, _ = binding.decay_forward(*qkv, g, SCALE, layout="bnhd")
    whole = after(x, o, h)
    prompt = x[:, :max(lengths)].contiguous()
    for b, n in enumerate(lengths):
        prompt[b, n:] = 0
    h, qkv = before(prompt)
    o, state = binding.decay_forward(*qkv, g, SCALE, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                                     want_state=True, layout="bnhd")
    outs = after(prompt, o, h)
    tol = 1e-5 if dtype == "f32" else 2.0 ** -5
    close = lambda a, b: (a.float() - b.float()).norm() <= tol * b.float().norm()   # noqa: E731
    for b, n in enumerate(lengths):
        assert all(close(a[b, :n], w[b, :n]) for a, w in zip(outs, whole))
    for step in range(6):
        at = [min(n + step, N - 1) for n in lengths]
        live = torch.tensor([n + step < N for n in lengths], dtype=torch.int32, device="cuda")
        token = torch.stack([x[b, t] for b, t in enumerate(at)]).unsqueeze(1)
        h, qkv = before(token)
        o = binding.decay_step(*(t[:, 0].contiguous() for t in qkv), g, state, SCALE, active=live)
        outs = after(token, o, h)
        for b, t in enumerate(at):
            if live[b]:
                assert all(close(a[b, 0], w[b, t]) for a, w in zip(outs, whole)), (step, b)
