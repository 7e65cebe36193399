"""The residual norm against its plain form in 64 bits, element by element.

Tolerances: outputs are rounded once (u: half a step of their type); before that everything is fp32, with sums over at most 8192
channels taken 16 a lane and then pairwise (at most 32 roundings).  An element of a normalised row is off by at most 2^-17 of its scale
times the magnitudes that went into it and into the row's mean, the more so the further out it lies; gradients, of the same
kind, by 2^-15 of theirs."""
import pytest
import torch

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.autograd import residual_norm
from paper_2508_12594_amd.binding import FlareError
from tests import _plain

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
PARAMS = ("pre_weight", "pre_bias", "post_weight", "post_bias")


def make(shape, dtype, x_f32, pre, post, gate, weights, biases, seed):
    gen = torch.Generator().manual_seed(seed)
    dt, C = TYPES[dtype], shape[-1]
    xt = torch.float32 if x_f32 else dt
    t = dict(x=(2 * torch.randn(shape, generator=gen) + 0.5).to(xt), y=torch.randn(shape, generator=gen).to(dt),
             dx_out=torch.randn(shape, generator=gen).to(xt), dh=torch.randn(shape, generator=gen).to(dt))
    gshape = {"none": None, "token": shape, "channel": (C,)}.get(gate, None) if gate != "item" else (shape[0],) + (1,) * (
        len(shape) - 2) + (C,)
    t["gate"] = None if gshape is None else (0.5 + torch.randn(gshape, generator=gen)).to(dt)
    for side, kind in (("pre", pre), ("post", post)):
        t[side + "_weight"] = 1 + 0.2 * torch.randn(C, generator=gen) if kind != "none" and weights else None
        t[side + "_bias"] = 0.2 * torch.randn(C, generator=gen) if kind != "none" and biases else None
    if pre == "none":
        t["dh"] = None
    return t


def rows_of(t, shape):
    """fp64 [rows,C], a shared gate repeated."""
    return None if t is None else (t.double().expand(shape) if t.dim() == 1 or t.shape != shape else t.double()).reshape(-1, shape[-1])


def near(name, got, want, tol, dtype):
    got = got.double().cpu().reshape(want.shape)
    tol = tol + UNIT[dtype] * want.abs() + TINY[dtype]
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).max().item()
    print("[case]    %s: worst error / tolerance %.3f" % (name, worst), flush=True)
    assert torch.isfinite(got).all() and worst <= 1.0, name


def sizes(w, p, s, pre, post, act, alpha, eps):
    """Magnitudes that went into u, x_out and h, and what a step of 2^-17 of them does to h."""
    mean = lambda t: t.mean(1, keepdim=True)   # noqa: E731
    mx = w["x"].abs()
    mu = None
    if w["y"] is not None:
        mu = w["y"].abs()
        if post != "none":
            mu = s["r_post"] * (mu + mean(mu)) * (1 + s["uh"].abs())
            mu = mu * (p["post_weight"].abs() if "post_weight" in p else 1) + (p["post_bias"].abs() if "post_bias" in p else 0)
        value = 1.0 if w["gate"] is None else _plain.act(w["gate"], act)[0].abs()
        mx = mx + alpha * value * mu
    mh = None
    if pre != "none":
        mh = s["r_pre"] * (mx + mean(mx)) * (1 + s["xh"].abs())
        mh = mh * (p["pre_weight"].abs() if "pre_weight" in p else 1) + (p["pre_bias"].abs() if "pre_bias" in p else 0)
    return mu, mx, mh


CASES = [  # shape, dtype, x_f32, pre, post, gate, act, weights, biases, alpha
    ((1, 64), "bf16", False, "layer", "none", "none", "none", True, True, 1.0),
    ((37, 64), "f16", False, "rms", "rms", "token", "silu", True, False, 0.5),
    ((2, 70, 128), "bf16", True, "layer", "layer", "item", "sigmoid", True, True, 1.0),
    ((5, 1, 128), "f32", False, "layer", "none", "item", "none", False, False, 1.0),
    ((3, 67, 200), "bf16", False, "rms", "layer", "channel", "none", True, True, -0.7),
    ((129, 256), "f32", False, "layer", "rms", "token", "sigmoid", True, True, 0.3),
    ((2, 33, 512), "f16", True, "none", "rms", "item", "silu", True, True, 1.0),
    ((9, 1000), "bf16", False, "layer", "layer", "token", "none", True, True, 1.0),
    ((17, 1024), "f32", False, "rms", "none", "none", "none", True, False, 2.0),
    ((4, 5, 2048), "bf16", True, "rms", "rms", "item", "silu", True, False, 0.5),
    ((21, 4096), "f16", False, "layer", "rms", "token", "silu", False, True, 0.5),
    ((7, 8192), "bf16", False, "layer", "layer", "channel", "sigmoid", True, True, 1.0),
    ((6, 8192), "f32", False, "rms", "rms", "token", "silu", True, True, 1.0),
    ((11, 1), "f32", False, "layer", "none", "none", "none", True, True, 1.0),
    ((50, 33), "bf16", False, "layer", "rms", "token", "silu", True, True, 1.0),
    ((3, 40, 250), "f32", False, "layer", "layer", "channel", "none", True, True, 1.0),
    ((2, 9, 513), "f16", True, "rms", "layer", "item", "sigmoid", True, True, 1.0),
    ((5, 2049), "bf16", False, "layer", "layer", "token", "silu", True, True, 1.0),
    ((3, 8191), "f32", False, "layer", "rms", "channel", "silu", True, True, 1.0),
    ((4000, 64), "bf16", False, "layer", "none", "channel", "none", True, True, 1.0),
    ((3, 2500, 72), "f32", False, "rms", "rms", "item", "none", True, False, 1.0),
    ((300, 2, 96), "f32", False, "layer", "none", "item", "silu", True, True, 1.0),
]


@pytest.mark.parametrize("shape,dtype,x_f32,pre,post,gate,act,weights,biases,alpha", CASES)
def test_forward_and_backward(shape, dtype, x_f32, pre, post, gate, act, weights, biases, alpha):
    print("[case] norm %s %s x_f32=%s pre=%s post=%s gate=%s %s" % (shape, dtype, x_f32, pre, post, gate, act), flush=True)
    eps = 1e-5
    t = make(shape, dtype, x_f32, pre, post, gate, weights, biases, sum(shape))
    dev = {n: None if a is None else a.cuda() for n, a in t.items()}
    w = {n: rows_of(a, shape) for n, a in t.items() if n not in PARAMS}
    p = {n: t[n].double() for n in PARAMS if t[n] is not None}
    kinds = dict(pre=pre, post=post, gate_act=act, alpha=alpha)
    rows = w["x"].shape[0]
    stats = torch.empty(rows, 4, device="cuda")
    given = {n: dev[n] for n in PARAMS}
    x_out, h = binding.residual_norm_forward(dev["x"], dev["y"], dev["gate"], eps=eps, stats=stats, **given, **kinds)
    want_x, want_h, s = _plain.residual_norm(w["x"], w["y"], w["gate"], p, pre, post, act, alpha, eps)
    mu, mx, mh = sizes(w, p, s, pre, post, act, abs(alpha), eps)
    near("x_out", x_out, want_x, 2.0 ** -17 * mx, x_out.dtype)
    assert x_out.dtype == dev["x"].dtype and x_out.shape == shape
    if pre == "none":
        assert h is None
    else:
        assert h.dtype == TYPES[dtype] and h.shape == shape
        near("h", h, want_h, 2.0 ** -17 * mh, h.dtype)

    grads = binding.residual_norm_backward(dev["x"], dev["y"], dev["dx_out"], dev["dh"], stats, gate=dev["gate"], **given, **kinds)
    got = dict(zip(("x", "y", "gate") + PARAMS, grads))
    want = _plain.residual_norm_gradients(w["x"], w["y"], w["gate"], p, pre, post, act, alpha, eps, w["dx_out"], w["dh"])
    # the same formulas over magnitudes
    mean = lambda a: a.mean(1, keepdim=True)   # noqa: E731

    def norm_size(d, unit, r, weight, m):
        # d: magnitude of the gradient coming in; m: magnitude that the row was normalised from
        d = d * (weight.abs() if weight is not None else 1)
        spread = 1 + r * (m + mean(m))                      # an error of the normalised row, in steps of its own size
        return r * (d + mean(d) + (1 + unit.abs()) * mean(d * (1 + unit.abs()) * spread)) * spread

    gx = w["dx_out"].abs()
    if pre != "none":
        gx = gx + norm_size(w["dh"].abs(), s["xh"], s["r_pre"], p.get("pre_weight"), mx)
    size = {"x": gx}
    d = abs(alpha) * gx
    if w["gate"] is not None:
        value, slope = _plain.act(w["gate"], act)
        # (sigmoid and 1 - sigmoid are good to a few steps of 1)
        size["gate"] = d * mu * (slope.abs() + (1 + w["gate"].abs() if act != "none" else 0))
        d = d * (value.abs() + (0.01 if act != "none" else 0))
    if post != "none":
        spread = 1 + s["r_post"] * (w["y"].abs() + mean(w["y"].abs()))
        size["post_weight"], size["post_bias"] = (d * (1 + s["uh"].abs()) * spread).sum(0), d.sum(0)
        size["y"] = norm_size(d, s["uh"], s["r_post"], p.get("post_weight"), w["y"].abs())
    else:
        size["y"] = d
    if pre != "none":
        spread = 1 + s["r_pre"] * (mx + mean(mx))
        size["pre_weight"], size["pre_bias"] = (w["dh"].abs() * (1 + s["xh"].abs()) * spread).sum(0), w["dh"].abs().sum(0)
    for n, g in got.items():
        if (dev[n] if n in dev else None) is None:
            assert g is None, n
            continue
        assert g.shape == dev[n].shape and g.dtype == dev[n].dtype
        a, m = want[n], size[n]
        if n == "gate" and gate in ("item", "channel"):
            per = shape[0] if gate == "item" else 1
            a, m = a.reshape(per, -1, shape[-1]).sum(1), m.reshape(per, -1, shape[-1]).sum(1)
        near("d" + n, g, a, 2.0 ** -15 * m, g.dtype)

    # the same bits again; outputs over the inputs
    again = binding.residual_norm_backward(dev["x"], dev["y"], dev["dx_out"], dev["dh"], stats, gate=dev["gate"], **given, **kinds)
    assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(grads, again))
    x, y = dev["x"].clone(), dev["y"].clone()
    x2, h2 = binding.residual_norm_forward(x, y, dev["gate"], eps=eps, x_out=x, h=None if pre == "none" else y, **given, **kinds)
    assert x2 is x and torch.equal(x, x_out) and (h is None or torch.equal(y, h))


@pytest.mark.parametrize("C,dtype,h_dtype", [(128, "bf16", None), (320, "f32", "f16"), (77, "f32", None)])
def test_norm_alone(C, dtype, h_dtype):
    """Before the first block there is no branch: h = pre(x), in a 16-bit type of its own if asked for."""
    print("[case] norm alone C%d %s -> %s" % (C, dtype, h_dtype), flush=True)
    t = make((3, 11, C), dtype, False, "layer", "none", "none", True, True, 3)
    x, weight, bias = t["x"].cuda(), t["pre_weight"].cuda(), t["pre_bias"].cuda()
    want = TYPES[h_dtype] if h_dtype else None
    x = x.requires_grad_(True)
    x_out, h = residual_norm(x, pre_weight=weight, pre_bias=bias, h_dtype=want)
    assert x_out is x and h.dtype == (want or x.dtype)
    p = dict(pre_weight=t["pre_weight"].double(), pre_bias=t["pre_bias"].double())
    w = {"x": rows_of(t["x"], (3, 11, C)), "y": None, "gate": None}
    _, ref, s = _plain.residual_norm(w["x"], None, None, p, "layer", "none", "none", 1.0, 1e-5)
    _, mx, mh = sizes(w, p, s, "layer", "none", "none", 1.0, 1e-5)
    near("h", h.detach(), ref, 2.0 ** -17 * mh, h.dtype)
    dh = t["dh"].cuda().to(h.dtype)
    dx, = torch.autograd.grad(h, x, dh)
    ref = _plain.residual_norm_gradients(w["x"], None, None, p, "layer", "none", "none", 1.0, 1e-5, None,
                                         dh.double().cpu().reshape(-1, C))["x"]
    near("dx", dx, ref, 2.0 ** -11 * ref.abs().max(), dx.dtype)


def test_autograd_forms():
    """Through autograd: the binding's gradients, whichever output is used, with strided inputs and saved-tensor hooks; refusals."""
    import torch.autograd.forward_ad as fwad
    print("[case] norm autograd", flush=True)
    shape = (2, 50, 128)
    t = {n: None if a is None else a.cuda() for n, a in make(shape, "bf16", False, "layer", "rms", "item", True, True, 5).items()}
    kinds = dict(pre="layer", post="rms", gate_act="silu", alpha=0.5)
    given = {n: t[n] for n in PARAMS}
    stats = torch.empty(100, 4, device="cuda")
    binding.residual_norm_forward(t["x"], t["y"], t["gate"], stats=stats, **given, **kinds)
    names = ("x", "y", "gate") + PARAMS
    leaves = {n: t[n].clone().requires_grad_(True) for n in names}
    leaves["y"] = t["y"].transpose(0, 1).contiguous().transpose(0, 1).requires_grad_(True)      # strided
    call = lambda: residual_norm(leaves["x"], leaves["y"], leaves["gate"], **{n: leaves[n] for n in PARAMS}, **kinds)   # noqa: E731
    for dx_out, dh in ((t["dx_out"], t["dh"]), (None, t["dh"]), (t["dx_out"], None)):
        want = binding.residual_norm_backward(t["x"], t["y"], dx_out, dh, stats, gate=t["gate"], **given, **kinds)
        x_out, h = call()
        used = [(o, d) for o, d in ((x_out, dx_out), (h, dh)) if d is not None]
        got = torch.autograd.grad([o for o, _ in used], list(leaves.values()), [d for _, d in used], allow_unused=True)
        for n, a, b in zip(names, got, want):
            assert torch.equal(a, b), n
    x_out, h = call()
    got, = torch.autograd.grad([x_out, h], leaves["gate"], [t["dx_out"], t["dh"]])       # only one gradient
    want = binding.residual_norm_backward(t["x"], t["y"], t["dx_out"], t["dh"], stats, gate=t["gate"], **given, **kinds)
    assert torch.equal(got, want[2])
    for which in range(8):
        count = [0]

        def unpack(a):
            count[0] += 1
            return a.flatten()[:-8].clone() if count[0] - 1 == which else a.clone()

        with torch.autograd.graph.saved_tensors_hooks(lambda a: a, unpack):
            x_out, h = call()
        with pytest.raises(FlareError):
            torch.autograd.grad([x_out, h], leaves["x"], [t["dx_out"], t["dh"]])
    with fwad.dual_level():
        with pytest.raises(FlareError):
            residual_norm(fwad.make_dual(t["x"], t["x"]), t["y"], **{n: t[n] for n in PARAMS}, **kinds)
    x = t["x"].clone().requires_grad_(True)
    held = residual_norm(x, t["y"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(FlareError):
            residual_norm(x, t["y"])
    del held


def test_traced_residual_norm_is_an_operation():
    print("[case] norm traced", flush=True)
    t = {n: None if a is None else a.cuda() for n, a in make((20, 64), "f32", False, "layer", "rms", "none", True, True, 7).items()}
    u = {n: None if a is None else a.cuda() for n, a in make((30, 64), "f32", False, "layer", "rms", "none", True, True, 8).items()}
    step = lambda x, y, w: residual_norm(x, y, post="rms", pre_weight=w)   # noqa: E731
    traced = torch.jit.trace(step, (t["x"], t["y"], t["pre_weight"]), check_trace=False)
    leaves = [u[n].clone().requires_grad_(True) for n in ("x", "y", "pre_weight")]
    got, want = traced(*leaves), step(*leaves)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for a, b in zip(*(torch.autograd.grad(o, leaves, [u["dx_out"], u["dh"]]) for o in (got, want))):
        assert torch.equal(a, b)


def test_gradients_are_differences():
    """Central differences of the forward, in fp32: the truncation falls with the square of the step, the rounding grows with its
    inverse; at 2^-6 of the inputs' size both are below 1e-3 of the loss's own size."""
    print("[case] norm differences", flush=True)
    shape = (6, 96)
    t = {n: a.cuda() for n, a in make(shape, "f32", False, "layer", "rms", "token", True, True, 9).items() if a is not None}
    names = ("x", "y", "gate") + PARAMS
    leaves = {n: t[n].clone().requires_grad_(True) for n in names}

    def loss(s):
        x_out, h = residual_norm(s["x"], s["y"], s["gate"], **{n: s[n] for n in PARAMS}, post="rms", gate_act="silu", alpha=0.5)
        return (x_out.double() * t["dx_out"].double()).sum() + (h.double() * t["dh"].double()).sum()

    grads = dict(zip(names, torch.autograd.grad(loss(leaves), list(leaves.values()))))
    gen = torch.Generator(device="cuda").manual_seed(2)
    for n in names:
        step = 2.0 ** -6 * torch.randn(leaves[n].shape, generator=gen, device="cuda")
        with torch.no_grad():
            up, down = (loss({**leaves, n: leaves[n] + sign * step}) for sign in (1, -1))
        want = (grads[n].double() * step.double()).sum()
        assert abs((up - down) / 2 - want) <= 1e-3 * (grads[n].double() * step.double()).norm() + 1e-6 * up.abs(), n


def test_many_rows_and_graph():
    """More rows than a launch has workgroups, a gate of each item, on another stream and captured: every replay the eager bits."""
    print("[case] norm graph", flush=True)
    shape = (3, 30001, 64)
    t = {n: None if a is None else a.cuda() for n, a in make(shape, "bf16", True, "layer", "rms", "item", True, True, 11).items()}
    given = {n: t[n] for n in PARAMS}
    kinds = dict(pre="layer", post="rms", gate_act="sigmoid")
    rows = shape[0] * shape[1]
    stats = torch.empty(rows, 4, device="cuda")
    x_out, h = binding.residual_norm_forward(t["x"], t["y"], t["gate"], stats=stats, **given, **kinds)
    grads = binding.residual_norm_backward(t["x"], t["y"], t["dx_out"], t["dh"], stats, gate=t["gate"], **given, **kinds)
    w = {n: rows_of(a, shape) for n, a in t.items() if n not in PARAMS}
    p = {n: t[n].double() for n in PARAMS if t[n] is not None}
    want = _plain.residual_norm_gradients(w["x"], w["y"], w["gate"], p, "layer", "rms", "sigmoid", 1.0, 1e-5, w["dx_out"], w["dh"])
    for n, g in zip(PARAMS, grads[3:]):            # sums of 90003 terms of about 1: 2^-15 of their magnitudes
        assert (g.double() - want[n]).abs().max() <= 2.0 ** -15 * 4 * rows, n
    per_item = want["gate"].reshape(3, -1, 64).sum(1)
    assert (grads[2].double().reshape(3, 64) - per_item).abs().max() <= 2.0 ** -15 * 4 * 30001 + 2.0 ** -8 * per_item.abs().max()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    x2, h2 = torch.empty_like(x_out), torch.empty_like(h)
    torch.cuda.synchronize()
    binding.residual_norm_forward(t["x"], t["y"], t["gate"], x_out=x2, h=h2, stream=side, **given, **kinds)
    grads2 = binding.residual_norm_backward(t["x"], t["y"], t["dx_out"], t["dh"], stats, gate=t["gate"], stream=side, **given, **kinds)
    torch.cuda.synchronize()
    assert torch.equal(x2, x_out) and torch.equal(h2, h) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.residual_norm_forward(t["x"], t["y"], t["gate"], x_out=x2, h=h2, **given, **kinds)
        grads2 = binding.residual_norm_backward(t["x"], t["y"], t["dx_out"], t["dh"], stats, gate=t["gate"], **given, **kinds)
    for _ in range(3):
        for a in (x2, h2) + grads2:
            a.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x2, x_out) and torch.equal(h2, h) and all(torch.equal(a, b) for a, b in zip(grads, grads2))


def test_offsets_beyond_32_bits():
    """More than 2^32 elements a tensor: the last rows."""
    print("[case] norm, 8.6 GB a tensor", flush=True)
    rows, C = (1 << 21) + 3, 2048
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.empty(rows, C, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    stats = torch.empty(rows, 4, device="cuda")
    tail = slice(rows - 5, rows)
    x_out, h = binding.residual_norm_forward(x, y, post="rms", alpha=0.5, stats=stats)
    small = binding.residual_norm_forward(x[tail].contiguous(), y[tail].contiguous(), post="rms", alpha=0.5)
    assert torch.equal(x_out[tail], small[0]) and torch.equal(h[tail], small[1])
    del h
    grads = binding.residual_norm_backward(x, y, x_out, None, stats, post="rms", alpha=0.5)
    small = binding.residual_norm_backward(x[tail].contiguous(), y[tail].contiguous(), x_out[tail].contiguous(), None,
                                           stats[tail].contiguous(), post="rms", alpha=0.5)
    assert torch.equal(grads[0][tail], small[0]) and torch.equal(grads[1][tail], small[1])
    del x, y, x_out, grads
    torch.cuda.empty_cache()
