"""The decay mixer against its plain form in 64 bits, element by element.

Tolerances: with A the same sum taken over magnitudes, the kernels round a product's weighted pair (u), or the state where it
meets a query (u), and the result (u), u half a step of the storage type; every other operation is fp32, at most N + 2 d + 256
of them in a row (the 256 covers a weight 2^x, whose exponent is rounded).  fp16 operands lie behind a power of two that the
wave shares, which costs 2^-24 of the largest sum at most."""
import threading

import pytest
import torch

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.autograd import decay_mixer
from paper_2508_12594_amd.binding import FlareError
from tests import _plain

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def make(B, H, N, d, dtype, seed, layout="bhnd", lengths=None, state=False, decays=None, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype]
    t = {n: (size * torch.randn(B, H, N, d, generator=gen)).to(dt) for n in ("q", "k", "v", "d_o")}
    g = decays if decays is not None else [-1.0 / (4.0 * 16.0 ** (h / max(1, H - 1))) for h in range(H)]
    t["log_decay"] = torch.tensor(g, dtype=torch.float32)
    t["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    for n in ("state", "dstate_out"):
        t[n] = torch.randn(B, H, d, d, generator=gen) if state else None
    order = (lambda a: a.transpose(1, 2).contiguous()) if layout == "bnhd" else (lambda a: a)
    dev = {n: None if a is None else (order(a) if n in ("q", "k", "v", "d_o") else a).cuda() for n, a in t.items()}
    wide = {n: None if a is None else a if n == "lengths" else a.double() for n, a in t.items()}
    return dev, wide


def back(t, layout):
    return (t.transpose(1, 2) if layout == "bnhd" else t).double().cpu()


def magnitudes(w):
    return {n: a if a is None or n in ("lengths", "log_decay") else a.abs() for n, a in w.items()}


def check(name, got, want, size, dtype, N, d, roundings):
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]
    tol = (roundings * u + (N + 2 * d + 256) * 2.0 ** -24) * size + 2.0 ** -24 * size.max()
    if dtype == "f16" and name.startswith(("state", "dstate")):
        tol = tol + 2.0 ** -21 * size                       # what is added to the state is good to 2^-22 of a term
    if dtype == "f16":
        tol = tol + 2.0 ** -25                              # the smallest step of an fp16 output
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).max().item() if got.numel() else 0.0
    print("[case]    %s: worst error / tolerance %.3f" % (name, worst), flush=True)
    assert torch.isfinite(got).all() and worst <= 1.0, name


CASES = [  # B, H, N, d, dtype, layout, lengths, state
    (1, 1, 1, 64, "bf16", "bhnd", None, False),
    (2, 3, 1, 16, "f32", "bnhd", [1, 0], True),
    (1, 2, 31, 32, "f16", "bhnd", None, True),
    (2, 2, 32, 128, "bf16", "bnhd", None, True),
    (1, 3, 33, 64, "f32", "bnhd", None, False),
    (1, 2, 257, 16, "bf16", "bhnd", None, True),
    (1, 2, 700, 128, "bf16", "bnhd", None, True),
    (1, 2, 600, 128, "f16", "bhnd", None, False),
    (1, 1, 519, 128, "f32", "bhnd", None, True),
    (1, 5, 1000, 32, "bf16", "bnhd", None, False),
    (1, 2, 777, 64, "f16", "bnhd", None, True),
    (5, 2, 300, 64, "bf16", "bhnd", [300, 0, 1, 256, 257], True),
    (4, 3, 770, 16, "f16", "bnhd", [512, 770, 33, 513], True),
    (3, 1, 530, 32, "f32", "bhnd", [0, 530, 300], False),
    (3, 2, 290, 128, "bf16", "bnhd", [32, -5, 1000], True),
    # more items than a wave has lanes, in segments: most of them empty, some items full, some without a token
    (130, 2, 500, 16, "bf16", "bnhd", [(37 * b * b) % 501 if b % 5 else 0 for b in range(130)], True),
    (70, 1, 450, 32, "f16", "bhnd", [450 if b == 69 else b % 3 for b in range(70)], True),
]


@pytest.mark.parametrize("B,H,N,d,dtype,layout,lengths,state", CASES)
def test_forward_and_backward(B, H, N, d, dtype, layout, lengths, state):
    print("[case] decay B%d H%d N%d d%d %s %s %s state=%s" % (B, H, N, d, dtype, layout, lengths, state), flush=True)
    dev, wide = make(B, H, N, d, dtype, 7 * N + d, layout, lengths, state)
    scale = d ** -0.5
    if lengths is not None:
        wide["lengths"] = wide["lengths"].clamp(0, N)
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    keep = dict(lengths=dev["lengths"], state=dev["state"], layout=layout)
    o, s = binding.decay_forward(*args, scale, want_state=True, **keep)
    dq, dk, dv, ds = binding.decay_backward(*args, dev["d_o"], scale, dstate_out=dev["dstate_out"], want_dstate=True, **keep)
    torch.cuda.synchronize()
    mag = magnitudes(wide)

    def forward(t):
        return _plain.decay(t["q"], t["k"], t["v"], t["log_decay"], scale, t["lengths"], t["state"])

    def backward(t):
        return _plain.decay_gradients(t["q"], t["k"], t["v"], t["log_decay"], t["d_o"], scale, t["lengths"], t["state"],
                                      t["dstate_out"])

    for name, got, want, size in zip(("o", "state"), (o, s), forward(wide), forward(mag)):
        tok = name == "o"
        check(name, back(got, layout if tok else "bhnd"), want, size, dtype if tok or dtype == "f16" else "f32", N, d, 2 if tok else 1)
    for name, got, want, size in zip(("dq", "dk", "dv", "dstate"), (dq, dk, dv, ds), backward(wide), backward(mag)):
        tok = name != "dstate"
        if dtype == "f16" and not tok:
            size = size + 2.0 ** -14 * size.max()           # a weight times a subnormal d_o
        check(name, back(got, layout if tok else "bhnd"), want, size, dtype if tok or dtype == "f16" else "f32", N, d, 2 if tok else 1)
    # the same bits again, and with a workspace and outputs of the caller's (the state over the one that came in, o over q)
    f_bytes, b_bytes, m_bytes = binding.decay_workspace_bytes(B, H, N, d, binding._dtype_code(dev["q"]), layout,
                                                               padded=lengths is not None)
    marks = torch.full((m_bytes // 4,), float("nan"), device="cuda")
    ws = torch.full((max(f_bytes, b_bytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    again = binding.decay_backward(*args, dev["d_o"], scale, dstate_out=dev["dstate_out"], want_dstate=True, workspace=ws, **keep)
    assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dv, ds)))
    carried = dev["state"].clone() if state else None
    over = dev["q"].clone()
    keep["state"] = carried
    o2, s2 = binding.decay_forward(over, *args[1:], scale, o=over, state_out=carried, want_state=True, workspace=ws, **keep)
    assert o2 is over and torch.equal(o2, o) and torch.equal(s2, s)
    keep["state"] = dev["state"]
    binding.decay_forward(*args, scale, marks=marks, **keep)
    again = binding.decay_backward(*args, dev["d_o"], scale, dstate_out=dev["dstate_out"], want_dstate=True, marks=marks, **keep)
    assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dv, ds)))
    if lengths is not None:      # padding is zeros
        for t in (o, dq, dk, dv):
            for b in range(B):
                assert (back(t, layout)[b, :, max(0, min(N, lengths[b])):] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_extreme_decays(dtype):
    """No decay at all, decays that leave nothing of the token before, a decay of -inf (only the token itself counts); a head whose log
    decay is above 0 or NaN is NaN, the others do not notice."""
    H, N, d = 7, 300, 32
    decays = [0.0, -1e-7, -20.0, -1000.0, float("-inf"), 0.5, float("nan")]
    dev, wide = make(1, H, N, d, dtype, 5, decays=decays, state=True)
    print("[case] extreme decays " + dtype, flush=True)
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    o, s = binding.decay_forward(*args, 0.2, state=dev["state"], want_state=True)
    grads = binding.decay_backward(*args, dev["d_o"], 0.2, state=dev["state"], dstate_out=dev["dstate_out"], want_dstate=True)
    tok = torch.empty(1, H, d, dtype=dev["q"].dtype, device="cuda")
    step_state = torch.empty_like(dev["state"])
    binding.decay_step(*(dev[n][:, :, 0].contiguous() for n in ("q", "k", "v")), dev["log_decay"], dev["state"], 0.2,
                       state_out=step_state, o=tok)
    for t in (o, s, tok, step_state) + grads:
        assert t[:, 5:].isnan().all() and t[:, :5].isfinite().all()
    five = {n: a[:5] if n == "log_decay" else None if a is None else a[:, :5] for n, a in wide.items()}
    want, size = (_plain.decay(t["q"], t["k"], t["v"], t["log_decay"], 0.2, None, t["state"]) for t in (five, magnitudes(five)))
    check("o", back(o, "bhnd")[:, :5], want[0], size[0], dtype, N, d, 2)
    check("state", back(s, "bhnd")[:, :5], want[1], size[1], dtype if dtype == "f16" else "f32", N, d, 1)


def test_padding_is_not_read():
    """Whatever lies behind an item's length, NaN and infinities too, is not looked at."""
    B, H, N, d = 3, 2, 400, 64
    print("[case] padding", flush=True)
    for dtype in ("bf16", "f32"):
        lengths = [17, 400, 300]
        dev, _ = make(B, H, N, d, dtype, 9, lengths=lengths, state=True)
        args = ("q", "k", "v", "log_decay")

        def everything(t):
            keep = dict(lengths=t["lengths"], state=t["state"])
            return binding.decay_forward(*(t[n] for n in args), 0.1, want_state=True, **keep) + binding.decay_backward(
                *(t[n] for n in args), t["d_o"], 0.1, dstate_out=t["dstate_out"], want_dstate=True, **keep)

        clean = everything(dev)
        spoiled = dict(dev)
        for n, bad in (("q", float("nan")), ("k", float("inf")), ("v", float("nan")), ("d_o", float("-inf"))):
            spoiled[n] = dev[n].clone()
            for b, n_b in enumerate(lengths):
                spoiled[n][b, :, n_b:] = bad
        assert all(torch.equal(a, b) for a, b in zip(everything(spoiled), clean))


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128), ("f16", 16)])
def test_pieces_and_single_tokens_make_the_whole(dtype, d):
    """A prompt in two pieces, then token by token: the states and outputs of one long call."""
    B, H, N = 2, 3, 90
    print("[case] pieces %s d%d" % (dtype, d), flush=True)
    dev, wide = make(B, H, N, d, dtype, 11)
    q, k, v, g = (dev[n] for n in ("q", "k", "v", "log_decay"))
    part = lambda a, z: [t[:, :, a:z].contiguous() for t in (q, k, v)]   # noqa: E731
    outs = []
    o, s = binding.decay_forward(*part(0, 37), g, 0.3, want_state=True)
    outs.append(o)
    o, _ = binding.decay_forward(*part(37, 70), g, 0.3, state=s, state_out=s)
    outs.append(o)
    for t in range(70, N):
        one = [x[:, :, 0].contiguous() for x in part(t, t + 1)]
        outs.append(binding.decay_step(*one, g, s, 0.3).unsqueeze(2))
    want, size = (_plain.decay(w["q"], w["k"], w["v"], w["log_decay"], 0.3) for w in (wide, magnitudes(wide)))
    check("o", back(torch.cat(outs, 2), "bhnd"), want[0], size[0], dtype, N, d, 2)
    check("state", back(s, "bhnd"), want[1], size[1], dtype if dtype == "f16" else "f32", N, d, 1)


@pytest.mark.parametrize("B,H,d,dtype", [(1, 1, 16, "bf16"), (3, 5, 32, "f32"), (2, 7, 64, "f16"), (1, 3, 128, "bf16"),
                                         (600, 1, 64, "bf16"), (65, 8, 128, "f32")])
def test_step(B, H, d, dtype):
    print("[case] step B%d H%d d%d %s" % (B, H, d, dtype), flush=True)
    dev, wide = make(B, H, 1, d, dtype, 3, state=True)
    tok = [dev[n][:, :, 0].contiguous() for n in ("q", "k", "v")]
    want, size = (_plain.decay(w["q"], w["k"], w["v"], w["log_decay"], 0.25, None, w["state"]) for w in (wide, magnitudes(wide)))
    out = torch.empty_like(dev["state"])
    o = binding.decay_step(*tok, dev["log_decay"], dev["state"], 0.25, state_out=out)
    check("o", back(o, "bhnd"), want[0][:, :, 0], size[0][:, :, 0], dtype, 1, d, 1)
    check("state", back(out, "bhnd"), want[1], size[1], "f32", 1, d, 1)
    active = torch.tensor([(b % 3) - 1 for b in range(B)], dtype=torch.int32, device="cuda")     # -1 and 0: none
    state = dev["state"].clone()
    o2 = binding.decay_step(*tok, dev["log_decay"], state, 0.25, active=active)
    on = active > 0
    assert torch.equal(state[on], out[on]) and torch.equal(state[~on], dev["state"][~on])
    assert torch.equal(o2[on], o[on]) and (o2[~on] == 0).all()


@pytest.mark.parametrize("q_size,kv_size,g_size", [(2.0 ** -10, 256.0, 2.0 ** -18), (1024.0, 2.0 ** -9, 2.0 ** -8)])
def test_fp16_beyond_its_range(q_size, kv_size, g_size):
    """A state above 65504, or one among the subnormals, and such gradients: nothing may overflow, or be lost, inside."""
    B, H, N, d = 1, 2, 500, 32
    print("[case] fp16 range %g" % kv_size, flush=True)
    dev, wide = make(B, H, N, d, "f16", 13, decays=[0.0, -0.001])
    for n, f in (("q", q_size), ("k", kv_size), ("v", kv_size), ("d_o", g_size)):
        dev[n] = (dev[n] * f).contiguous()
        wide[n] = dev[n].double().cpu()
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    want, size = (_plain.decay(t["q"], t["k"], t["v"], t["log_decay"], 2.0 ** -6) for t in (wide, magnitudes(wide)))
    o, s = binding.decay_forward(*args, 2.0 ** -6, want_state=True)
    assert s.abs().max() > 65504 or s.abs().max() < 2.0 ** -10
    check("o", back(o, "bhnd"), want[0], size[0], "f16", N, d, 2)
    check("state", back(s, "bhnd"), want[1], size[1], "f16", N, d, 1)
    grads = binding.decay_backward(*args, dev["d_o"], 2.0 ** -6)
    want, size = (_plain.decay_gradients(t["q"], t["k"], t["v"], t["log_decay"], t["d_o"], 2.0 ** -6)
                  for t in (wide, magnitudes(wide)))
    for name, a, b, m in zip(("dq", "dk", "dv"), grads, want, size):
        check(name, back(a, "bhnd"), b, m, "f16", N, d, 2)


def test_gradients_are_differences():
    """The mixer is linear in each of its tensors: a difference along any direction is the gradient's product with it."""
    B, H, N, d = 2, 2, 300, 32
    print("[case] differences", flush=True)
    dev, _ = make(B, H, N, d, "f32", 17, lengths=[300, 123], state=True)
    leaves = {n: dev[n].clone().requires_grad_(True) for n in ("q", "k", "v", "state")}

    def loss(t):
        o, s = decay_mixer(t["q"], t["k"], t["v"], dev["log_decay"], 0.2, lengths=dev["lengths"], state=t["state"], want_state=True)
        return (o.double() * dev["d_o"].double()).sum() + (s.double() * dev["dstate_out"].double()).sum()

    grads = dict(zip(leaves, torch.autograd.grad(loss(leaves), list(leaves.values()))))
    gen = torch.Generator(device="cuda").manual_seed(1)
    for n in leaves:
        step = torch.randn(leaves[n].shape, generator=gen, device="cuda")
        with torch.no_grad():
            up, down = (loss({**leaves, n: leaves[n] + sign * step}) for sign in (1, -1))
        want = (grads[n].double() * step.double()).sum()
        # every sum is of fp32 terms: random errors of 2^-24 of the largest partial results
        size = (grads[n].double() * step.double()).norm() + up.abs() + down.abs()
        assert abs((up - down) / 2 - want) <= 1e-4 * size, n


def test_autograd_forms():
    """Strided inputs, an unused output, saved-tensor hooks, threads; what is refused."""
    import torch.autograd.forward_ad as fwad
    print("[case] autograd forms", flush=True)
    B, H, N, d = 2, 4, 150, 32
    dev, _ = make(B, H, N, d, "bf16", 21, layout="bnhd", state=True)
    fused = torch.stack([dev[n] for n in ("q", "k", "v")], 2).requires_grad_(True)      # [B,N,3,H,d]: one projection's output
    g, scale = dev["log_decay"], 0.2

    def grads(which):
        q, k, v = fused.unbind(2)
        o, s = decay_mixer(q, k, v, g, scale, state=dev["state"], want_state=True, layout="bnhd")
        outs = {"o": [o], "state": [s], "both": [o, s]}[which]
        return torch.autograd.grad(outs, fused, [{id(o): dev["d_o"], id(s): dev["dstate_out"]}[id(t)] for t in outs])[0]

    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    for which in ("o", "state", "both"):
        zero = torch.zeros_like(dev["d_o"])
        want = binding.decay_backward(*args, zero if which == "state" else dev["d_o"], scale, state=dev["state"],
                                      dstate_out=None if which == "o" else dev["dstate_out"], layout="bnhd")[:3]
        assert torch.equal(grads(which), torch.stack(want, 2)), which
    want = grads("both")
    got = [None] * 3
    threads = [threading.Thread(target=lambda i=i: got.__setitem__(i, grads("both"))) for i in range(3)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in got)

    packed = []
    q = dev["q"].clone().requires_grad_(True)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: packed.append(t) or t, lambda t: t.clone()):
        o, none = decay_mixer(q, dev["k"], dev["v"], g, scale, layout="bnhd")
    assert none is None and len(packed) == 4
    torch.autograd.grad(o, q, dev["d_o"], retain_graph=True)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.flatten()[:-16].clone()):
        o, _ = decay_mixer(q, dev["k"], dev["v"], g, scale, layout="bnhd")
    with pytest.raises(FlareError):
        torch.autograd.grad(o, q, dev["d_o"])
    with pytest.raises(FlareError):
        decay_mixer(q, dev["k"], dev["v"], g.clone().requires_grad_(True), scale, layout="bnhd")
    with fwad.dual_level():
        with pytest.raises(FlareError):
            decay_mixer(fwad.make_dual(dev["q"], torch.ones_like(dev["q"])), dev["k"], dev["v"], g, scale, layout="bnhd")


def test_traced_decay_mixer_is_an_operation():
    print("[case] decay traced", flush=True)
    dev, _ = make(1, 2, 70, 32, "bf16", 23, state=True)
    other, _ = make(1, 2, 90, 32, "bf16", 24, state=True)
    step = lambda q, k, v, g, s: decay_mixer(q, k, v, g, 0.2, state=s, want_state=True)   # noqa: E731
    names = ("q", "k", "v", "log_decay", "state")
    traced = torch.jit.trace(step, [dev[n] for n in names], check_trace=False)
    leaves = [other[n].clone().requires_grad_(n != "log_decay") for n in names]
    got, want = traced(*leaves), step(*leaves)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    inputs = [t for t in leaves if t.requires_grad]
    for a, b in zip(*(torch.autograd.grad(x, inputs, [other["d_o"], other["dstate_out"]]) for x in (got, want))):
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    """More than 2^32 elements a tensor: the last tokens of the last head, which fast decays make independent of the others."""
    B, H, N, d = 2, 8, (1 << 21) + 5, 128
    print("[case] decay, 8.6 GB a tensor", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.empty(B, H, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    for t in (q, k, v):
        for b in range(B):
            t[b].normal_(generator=gen)
    g = torch.full((H,), -1.0, device="cuda")
    o, s = binding.decay_forward(q, k, v, g, 0.1, want_state=True)
    tail = {n: t[:, :, -64:].double().cpu() for n, t in (("q", q), ("k", k), ("v", v))}
    wide = dict(tail, log_decay=g.double().cpu())
    want, size = (_plain.decay(t["q"], t["k"], t["v"], t["log_decay"], 0.1) for t in (wide, magnitudes(wide)))
    check("o", o[:, :, -16:].double().cpu(), want[0][:, :, -16:], size[0][:, :, -16:], "bf16", 64, d, 2)
    check("state", s.double().cpu(), want[1], size[1], "f32", 64, d, 1)
    del q, k, v, o
    torch.cuda.empty_cache()


def test_other_stream_and_graph():
    """Forward, backward and step on another stream, and captured: every replay the eager bits."""
    print("[case] decay graph", flush=True)
    B, H, N, d = 2, 3, 700, 64
    dev, _ = make(B, H, N, d, "bf16", 31, lengths=[700, 400], state=True)
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    tok = [dev[n][:, :, 5].contiguous() for n in ("q", "k", "v")]
    f_bytes, b_bytes, _ = binding.decay_workspace_bytes(B, H, N, d, binding.FLARE_BF16, padded=True)
    assert f_bytes > 0 and b_bytes > 0
    ws = torch.empty(max(f_bytes, b_bytes), dtype=torch.uint8, device="cuda")

    def run(o, stream=None, workspace=None):
        keep = dict(lengths=dev["lengths"], state=dev["state"], workspace=workspace, stream=stream)
        binding.decay_forward(*args, 0.2, o=o["o"], state_out=o["state"], **keep)
        binding.decay_backward(*args, dev["d_o"], 0.2, dstate_out=dev["dstate_out"], dq=o["dq"], dk=o["dk"], dv=o["dv"],
                               dstate=o["dstate"], **keep)
        binding.decay_step(*tok, dev["log_decay"], dev["state"], 0.2, state_out=o["next"], o=o["token"], stream=stream)

    def buffers():
        o = {n: torch.full_like(dev["q"], float("nan")) for n in ("o", "dq", "dk", "dv")}
        o.update({n: torch.full_like(dev["state"], float("nan")) for n in ("state", "dstate", "next")})
        o["token"] = torch.full_like(tok[0], float("nan"))
        return o

    eager = buffers()
    run(eager)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = buffers()
    torch.cuda.synchronize()
    run(out, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(out[n], eager[n]) for n in out)
    with torch.cuda.stream(side):
        run(out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, workspace=ws)
    for _ in range(3):
        for t in out.values():
            t.fill_(float("nan"))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], eager[n]) for n in out)


def test_capture_beside_an_eager_graph_is_refused():
    """The gradient accumulators of leaves that an eager graph holds belong to the eager stream: the forward says so instead of the
    process ending in the backward.  Without that graph the capture works and replays."""
    print("[case] capture beside an eager graph", flush=True)
    dev, _ = make(1, 2, 100, 32, "bf16", 37)
    q, k, v = (dev[n].clone().requires_grad_(True) for n in ("q", "k", "v"))
    o, _ = decay_mixer(q, k, v, dev["log_decay"], 0.2)
    want = torch.autograd.grad(o, (q, k, v), dev["d_o"], retain_graph=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(FlareError):
            decay_mixer(q, k, v, dev["log_decay"], 0.2)
    del o
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(decay_mixer(q, k, v, dev["log_decay"], 0.2)[0], (q, k, v), dev["d_o"])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(decay_mixer(q, k, v, dev["log_decay"], 0.2)[0], (q, k, v), dev["d_o"])
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
