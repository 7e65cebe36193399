"""Timed cases of the decay mixer (causal linear attention with a decay for each head: whole prompts, training,
single tokens) and of the residual norm (the norms before and after a block, its gate and its residual scale in one
pass), from the smallest calls to the largest.

With own = False, run() computes the operators from elementary torch operations in 32 bits; with own = True it makes the calls
that a program makes of this package.  A case is a dict of plain values:
  op      "step":    binding.decay_step, one token for each item against its state (a generation loop)
          "prompt":  binding.decay_forward, a batch of prompts (serving)
          "train":   autograd.decay_mixer and the gradients of q, k, v (and the carried state)
          "norm":    binding.residual_norm_forward (inference)
          "norm-train": autograd.residual_norm and the gradients of everything it was given
  B, N, dtype  batch items, tokens per item, "bf16", "f16" or "f32"
 decay mixer:
  H, d    heads, head dimension
  layout  order of the token tensors: "bhnd" or "bnhd" (what a block's linear layers write)
  ragged  whether the batch is padded (item lengths between 0 and N)
  state   whether a state comes in and goes out (later pieces of a long sequence)
  reach   how many tokens the slowest head looks back; the fastest looks back 4
 residual norm:
  C       channels
  x_f32   whether the residual stream is kept in fp32 beside 16-bit branches
  pre, post    "none", "layer" or "rms": the norm after the addition and the norm of the branch
  gate    "none", "token" (a gate of its own for each token), "item" (one for each batch item) or "channel" (one for all)
  act     "none", "sigmoid" or "silu": what the gate goes through
  alpha   the residual scale
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5


def _decay(name, op, B, H, N, d, dtype, layout="bhnd", ragged=False, state=False, reach=256):
    c = dict(op=op, B=B, H=H, N=N, d=d, dtype=dtype, layout=layout, ragged=ragged, state=state, reach=reach)
    return dict(c, name=name) if name else c


def _norm(name, op, B, N, C, dtype, x_f32=False, pre="layer", post="none", gate="none", act="none", alpha=1.0):
    c = dict(op=op, B=B, N=N, C=C, dtype=dtype, x_f32=x_f32, pre=pre, post=post, gate=gate, act=act, alpha=alpha)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One stream of a generation loop: the smallest call, nothing but latency.
        _decay("step-one-stream", "step", 1, 8, 1, 64, "bf16", state=True),
        # A full serving batch, one token each: the states are read and written once.
        _decay("step-batch", "step", 128, 16, 1, 128, "bf16", state=True, reach=1024),
        # The second piece of a short prompt: an odd length, a state in and out.
        _decay("prompt-short", "prompt", 1, 8, 333, 64, "bf16", layout="bnhd", state=True),
        # A padded batch of prompts of different lengths, in the order the projections write, its states kept.
        _decay("prompt-ragged-f16", "prompt", 8, 16, 4097, 128, "f16", layout="bnhd", ragged=True, state=True, reach=1024),
        # One very long prompt.
        _decay("prompt-long", "prompt", 1, 16, 131072, 128, "bf16", layout="bnhd", reach=8192),
        # A batch of 4k-token sequences for classification (the mixer's own third workload), causal.
        _decay("train-sequences", "train", 32, 8, 4096, 32, "bf16"),
        # Single-precision training on sequences of an odd length.
        _decay("train-f32", "train", 2, 8, 10007, 64, "f32", reach=512),
        # Training on long sequences with wide heads, in pieces that hand their state on.
        _decay("train-long", "train", 1, 16, 32768, 128, "bf16", layout="bnhd", state=True, reach=4096),
        # Between two blocks of a generation loop: a norm on both sides of the addition.
        _norm("norm-tokens", "norm", 4, 1, 2048, "bf16", pre="rms", post="rms"),
        # The pre-norm residual of a block on a million points with 128 channels (the mixer's own fourth workload).
        _norm("norm-mesh", "norm", 1, 1000000, 128, "bf16"),
        # Single-precision training with an odd number of channels and a learned scale for each.
        _norm("norm-train-f32", "norm-train", 3, 5001, 250, "f32", post="layer", gate="channel"),
        # Training of a wide model: norms on both sides, a gate for each token, a residual scale.
        _norm("norm-train-wide", "norm-train", 4, 4096, 4096, "bf16", pre="rms", post="rms", gate="token", act="silu",
              alpha=0.5),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case: sizes over their whole range (logarithmically), mostly not multiples of anything."""
    op = rng.choice(["step", "prompt", "prompt", "train", "train", "norm", "norm-train", "norm-train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("step", "prompt", "train"):
        d = rng.choice([16, 32, 64, 64, 128])
        H = rng.choice([1, 4, 6, 8, 12, 16, 32])
        reach = _log_uniform(rng, 16, 16384)
        if op == "step":
            B = min(_log_uniform(rng, 1, 256), max(1, 33554432 // (H * d * d)))
            return _decay(None, op, B, H, 1, d, dtype, state=True, ragged=rng.random() < 0.25, reach=reach)
        B = rng.choice([1, 1, 2, 3, 8, _log_uniform(rng, 1, 64)])
        most = (2 ** 28 if op == "prompt" else 2 ** 26) // (4 if dtype == "f32" else 1)
        N = min(_log_uniform(rng, 1, 262144), max(1, most // (B * H * d)))
        return _decay(None, op, B, H, N, d, dtype, rng.choice(["bhnd", "bnhd"]), B > 1 and rng.random() < 0.4,
                      rng.random() < 0.4, reach)
    C = rng.choice([64, 128, 256, 512, 1024, 2048, 4096, 8192, _log_uniform(rng, 32, 8192), _log_uniform(rng, 32, 8192)])
    B = rng.choice([1, 2, 4, _log_uniform(rng, 1, 64)])
    most = (2 ** 27 if op == "norm" else 2 ** 26) // (2 if dtype == "f32" else 1)
    N = min(_log_uniform(rng, 1, 1000000), max(1, most // (B * C)))
    pre, post = rng.choice([("layer", "none"), ("rms", "none"), ("layer", "layer"), ("rms", "rms"), ("none", "rms")])
    gate = rng.choice(["none", "none", "token", "item", "channel"])
    act = "none" if gate in ("none", "channel") else rng.choice(["none", "sigmoid", "silu"])
    return _norm(None, op, B, N, C, dtype, dtype != "f32" and rng.random() < 0.3, pre, post, gate, act,
                 rng.choice([1.0, 1.0, 0.5, 1 / math.sqrt(8)]))


def _lengths(c):
    """Item lengths of a padded batch: the longest fills it, the others are anything, an empty one among many."""
    if not c["ragged"]:
        return [c["N"]] * c["B"]
    rng = random.Random(c["B"] * 1000003 + c["N"])
    out = [c["N"]] + [rng.randint(0, c["N"]) for _ in range(c["B"] - 1)]
    if c["B"] >= 8:
        out[rng.randrange(1, c["B"])] = 0
    rng.shuffle(out)
    return out


def _log_decays(c):
    H = c["H"]
    return [-1.0 / (4.0 * (c["reach"] / 4.0) ** (h / max(1, H - 1))) for h in range(H)]


def _prepare_decay(c, gen):
    B, H, N, d = (c[x] for x in "BHNd")
    dt = DTYPES[c["dtype"]]
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    shape = (B, H, d) if c["op"] == "step" else (B, H, N, d) if c["layout"] == "bhnd" else (B, N, H, d)
    s = dict(c, scale=1.0 / math.sqrt(d))
    for name in ("q", "k", "v"):      # projections behind a normalisation
        s[name] = randn(*shape).to(dt)
    s["log_decay"] = torch.tensor(_log_decays(c), dtype=torch.float32, device="cuda")
    s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
    s["state_in"] = None
    if c["state"]:                    # what the head's earlier tokens have left: its reach in random terms
        size = torch.sqrt(-0.5 / s["log_decay"]).view(1, H, 1, 1)
        s["state_in"] = randn(B, H, d, d) * size
        s["state_out"] = torch.empty_like(s["state_in"])
    if c["op"] == "train":
        s["do"] = randn(*shape).to(dt)
        s["dstate_out"] = 0.1 * randn(B, H, d, d) if c["state"] else None
        for name in ("q", "k", "v") + (("state_in",) if c["state"] else ()):
            s[name].requires_grad_(True)
    return s


def _prepare_norm(c, gen):
    B, N, C = c["B"], c["N"], c["C"]
    dt = DTYPES[c["dtype"]]
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    s = dict(c)
    # a residual stream has drifted off zero and has a few loud channels
    loud = 1.0 + 4.0 * (torch.rand((C,), generator=gen, device="cuda") < 0.02).float()
    s["x"] = (2.0 * randn(B, N, C) * loud + 0.5).to(torch.float32 if c["x_f32"] else dt)
    s["y"] = randn(B, N, C).to(dt)
    gate_shape = {"none": None, "token": (B, N, C), "item": (B, 1, C), "channel": (C,)}[c["gate"]]
    s["gate_in"] = None if gate_shape is None else (0.5 + randn(*gate_shape)).to(dt)
    for side in ("pre", "post"):
        kind = c[side]
        s[side + "_weight"] = None if kind == "none" else 1.0 + 0.1 * randn(C)
        s[side + "_bias"] = 0.1 * randn(C) if kind == "layer" else None
    if c["op"] == "norm-train":
        s["dx_out"] = randn(B, N, C).to(s["x"].dtype)
        s["dh"] = randn(B, N, C).to(dt) if c["pre"] != "none" else None
        for name in _norm_leaves(s):
            s[name].requires_grad_(True)
    return s


def _norm_leaves(s):
    names = ("x", "y", "gate_in", "pre_weight", "pre_bias", "post_weight", "post_bias")
    return [n for n in names if s[n] is not None]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_norm if c["op"].startswith("norm") else _prepare_decay)(c, gen)


# ---- the plain forms -----------------------------------------------------------------------------------------------
def _plain_decay(q, k, v, log_decay, scale, lengths, state):
    """[B,H,N,d] fp32 in chunks of 128 tokens; a token behind an item's end adds nothing and lets nothing decay."""
    B, H, N, d = q.shape
    at = torch.arange(1, N + 1, device=q.device, dtype=torch.float64)
    if lengths is None:
        age = at.view(1, 1, N).expand(B, 1, N)
        inside = None
    else:
        age = torch.minimum(at.view(1, N), lengths.double().view(B, 1)).view(B, 1, N)
        inside = (at.view(1, N) <= lengths.double().view(B, 1)).float().view(B, 1, N, 1)
        k = k * inside
    total = age * log_decay.double().view(1, H, 1)           # log of the decay since the sequence's start
    if state is None:
        state = torch.zeros((B, H, d, d), device=q.device)
    outs, before = [], torch.zeros((B, H, 1), device=q.device, dtype=torch.float64)
    for a in range(0, N, 128):
        z = min(a + 128, N)
        g = total[:, :, a:z]
        qc, kc, vc = q[:, :, a:z] * scale, k[:, :, a:z], v[:, :, a:z]
        gap = g.unsqueeze(3) - g.unsqueeze(2)
        past = torch.ones((z - a, z - a), device=q.device, dtype=torch.bool).tril()
        weight = torch.where(past, gap, torch.full_like(gap, -math.inf)).exp().float()
        out = torch.matmul(torch.matmul(qc, kc.transpose(2, 3)) * weight, vc)
        out = out + torch.matmul(qc, state) * (g - before).exp().float().unsqueeze(3)
        outs.append(out if inside is None else out * inside[:, :, a:z])
        end = g[:, :, -1:]
        state = state * (end - before).exp().float().unsqueeze(3) + torch.matmul(
            (kc * (end - g).exp().float().unsqueeze(3)).transpose(2, 3), vc)
        before = end
    return torch.cat(outs, 2), state


def _plain_step(s):
    q, k, v, state = s["q"].float(), s["k"].float(), s["v"].float(), s["state_in"]
    new = state * s["log_decay"].exp().view(1, -1, 1, 1) + k.unsqueeze(3) * v.unsqueeze(2)
    out = s["scale"] * (q.unsqueeze(3) * new).sum(2)
    if s["lengths"] is not None:
        active = (s["lengths"] > 0).view(-1, 1, 1)
        out = torch.where(active, out, torch.zeros_like(out))
        new = torch.where(active.unsqueeze(3), new, state)
    return {"o": out.to(s["q"].dtype), "state": new}


def _plain_one_norm(t, kind, weight, bias):
    if kind == "none":
        return t
    if kind == "layer":
        t = t - t.mean(2, keepdim=True)
    t = t * torch.rsqrt((t * t).mean(2, keepdim=True) + EPS)
    if weight is not None:
        t = t * weight
    return t if bias is None else t + bias


def _plain_norm(s):
    branch = _plain_one_norm(s["y"].float(), s["post"], s["post_weight"], s["post_bias"])
    if s["gate_in"] is not None:
        g = s["gate_in"].float()
        branch = branch * (g if s["act"] == "none" else torch.sigmoid(g) if s["act"] == "sigmoid" else g * torch.sigmoid(g))
    x = s["x"].float() + s["alpha"] * branch
    h = None if s["pre"] == "none" else _plain_one_norm(x, s["pre"], s["pre_weight"], s["pre_bias"]).to(s["y"].dtype)
    return x.to(s["x"].dtype), h


# ---- one pass ------------------------------------------------------------------------------------------------------
def _run_decay(s):
    op, lengths, scale = s["op"], s["lengths"], s["scale"]
    if own:
        from paper_2508_12594_amd import binding
        from paper_2508_12594_amd.autograd import decay_mixer
        if op == "step":
            o = binding.decay_step(s["q"], s["k"], s["v"], s["log_decay"], s["state_in"], scale, state_out=s["state_out"],
                                   active=lengths)
            return {"o": o, "state": s["state_out"]}
        if op == "prompt":
            o, state = binding.decay_forward(s["q"], s["k"], s["v"], s["log_decay"], scale, lengths=lengths,
                                             state=s["state_in"], state_out=s.get("state_out"), layout=s["layout"])
        else:
            o, state = decay_mixer(s["q"], s["k"], s["v"], s["log_decay"], scale, lengths=lengths, state=s["state_in"],
                                   want_state=s["state"], layout=s["layout"])
    elif op == "step":
        return _plain_step(s)
    else:
        bhnd = s["layout"] == "bhnd"
        order = (lambda t: t) if bhnd else (lambda t: t.transpose(1, 2))
        o, state = _plain_decay(*(order(s[n]).float() for n in ("q", "k", "v")), s["log_decay"], scale, lengths,
                                s["state_in"])
        o = order(o).to(s["q"].dtype)
    out = {"o": o}
    if s["state"]:
        out["state"] = state
    if op == "train":
        leaves = ["q", "k", "v"] + (["state_in"] if s["state"] else [])
        results, grads = ((o, state), (s["do"], s["dstate_out"])) if s["state"] else ((o,), (s["do"],))
        for name, g in zip(leaves, torch.autograd.grad(results, [s[n] for n in leaves], grads)):
            out["d" + name] = g
    return out


def _run_norm(s):
    if own:
        from paper_2508_12594_amd import binding
        from paper_2508_12594_amd.autograd import residual_norm
        args = dict(gate=s["gate_in"], pre=s["pre"], post=s["post"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"],
                    post_weight=s["post_weight"], post_bias=s["post_bias"], gate_act=s["act"], alpha=s["alpha"], eps=EPS)
        if s["op"] == "norm":
            x, h = binding.residual_norm_forward(s["x"], s["y"], **args)
        else:
            x, h = residual_norm(s["x"], s["y"], **args)
    else:
        x, h = _plain_norm(s)
    out = {"x": x} if h is None else {"x": x, "h": h}
    if s["op"] == "norm-train":
        leaves = _norm_leaves(s)
        results, grads = ((x,), (s["dx_out"],)) if h is None else ((x, h), (s["dx_out"], s["dh"]))
        for name, g in zip(leaves, torch.autograd.grad(results, [s[n] for n in leaves], grads)):
            out["d" + name] = g
    return out


def run(state):
    return (_run_norm if state["op"].startswith("norm") else _run_decay)(state)


# ---- the least a pass can read, write and compute --------------------------------------------------------------------
def work(case):
    c = case
    elem = 4 if c["dtype"] == "f32" else 2
    if c["op"].startswith("norm"):
        rows = c["B"] * c["N"]
        x = 4 if c["x_f32"] else elem
        gates = {"none": 0, "token": rows, "item": c["B"], "channel": 1}[c["gate"]]
        params = sum({"none": 0, "rms": 1, "layer": 2}[c[side]] for side in ("pre", "post"))
        h = 0 if c["pre"] == "none" else elem
        forward = c["C"] * (rows * (2 * x + elem + h) + gates * elem + params * 4)
        if c["op"] == "norm":
            return {"bytes": forward, "flops": 20.0 * rows * c["C"]}
        # x, y, the gate and the gradients of both outputs in; the gradients of all that was given out
        backward = c["C"] * (rows * (3 * x + 2 * elem + h) + 2 * gates * elem + 2 * params * 4)
        return {"bytes": forward + backward, "flops": 60.0 * rows * c["C"]}
    B, H, N, d = (c[x] for x in "BHNd")
    states = 4 * B * H * d * d if c["state"] else 0
    if c["op"] == "step":
        live = sum(1 for n in _lengths(c) if n) if c["ragged"] else B
        return {"bytes": 2 * states + 4 * B * H * d * elem, "flops": 5.0 * live * H * d * d}
    read, written = sum(_lengths(c)) * H * d * elem, B * N * H * d * elem
    term = H * d * sum(n * min(d, (n + 1) / 2) for n in _lengths(c))     # a product with the state, or with all pairs
    bytes_, flops = 3 * read + written + 2 * states, 4.0 * term
    if c["op"] == "train":
        bytes_ += 4 * read + 3 * written + 3 * states
        flops += 10.0 * term
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions, in 64 bits -------------------------------------------------------------------------------------
def _exact_pairs(a, b, c, rate, wanted, reverse=False):
    """out[i] = sum_j exp(-rate |i-j|) <a_i, b_j> c_j over j <= i (or j >= i), [N,d] fp64, for one head of one item: block by
    block of 2048 x 2048 pairs, leaving out blocks that are further apart than 64-bit weights reach."""
    N = a.shape[0]
    out = torch.zeros((wanted, c.shape[1]), dtype=torch.float64, device=a.device)
    size = 2048
    for i in range(0, N, size):
        ai = a[i:i + size]
        ti = torch.arange(i, i + ai.shape[0], device=a.device, dtype=torch.float64).view(-1, 1)
        for j in range(i, N, size) if reverse else range(i, -1, -size):
            if rate * (abs(i - j) - size) > 60.0:
                break
            bj, cj = b[j:j + size], c[j:j + size]
            tj = torch.arange(j, j + bj.shape[0], device=a.device, dtype=torch.float64).view(1, -1)
            gap = tj - ti if reverse else ti - tj
            weight = torch.exp(-rate * gap.clamp(min=0)) * (gap >= 0)
            out[i:i + ai.shape[0]] += (weight * (ai @ bj.T)) @ cj
    return out


def _exact_decay(c, s):
    B, H, N, d = (c[x] for x in "BHNd")
    heads_first = c["layout"] == "bhnd"
    wide = {n: s[n].detach().double() for n in ("q", "k", "v", "do", "state_in", "dstate_out") if s.get(n) is not None}
    lens, scale = _lengths(c), s["scale"]
    rates = [-x for x in s["log_decay"].double().tolist()]
    if c["op"] == "step":
        o, state = torch.zeros_like(wide["q"]), wide["state_in"].clone()
        for b in range(B):
            for h in range(H):
                if lens[b] > 0:
                    state[b, h] = math.exp(-rates[h]) * state[b, h] + torch.outer(wide["k"][b, h], wide["v"][b, h])
                    o[b, h] = scale * (state[b, h].T @ wide["q"][b, h])
        return {"o": o, "state": state}
    names = ["o"] + (["dq", "dk", "dv"] if c["op"] == "train" else [])
    out = {n: torch.zeros_like(wide["q"]) for n in names}
    if c["state"]:
        out["state"] = torch.zeros((B, H, d, d), dtype=torch.float64, device="cuda")
        if c["op"] == "train":
            out["dstate_in"] = torch.zeros_like(out["state"])
    for b in range(B):
        n = lens[b]
        for h in range(H):
            at = (b, h, slice(0, n)) if heads_first else (b, slice(0, n), h)
            rate = rates[h]
            q, k, v = (wide[x][at].contiguous() for x in ("q", "k", "v"))
            since = torch.exp(-rate * torch.arange(1, n + 1, device="cuda", dtype=torch.float64)).view(-1, 1)
            left = torch.exp(-rate * torch.arange(n - 1, -1, -1, device="cuda", dtype=torch.float64)).view(-1, 1)
            o = _exact_pairs(q, k, v, rate, n)
            if c["state"]:
                s0 = wide["state_in"][b, h]
                o += since * (q @ s0)
                out["state"][b, h] = math.exp(-rate * n) * s0 + (left * k).T @ v
            out["o"][at] = scale * o
            if c["op"] == "train":
                do = wide["do"][at].contiguous()
                dq = _exact_pairs(do, v, k, rate, n)
                dk = scale * _exact_pairs(v, do, q, rate, n, reverse=True)
                dv = scale * _exact_pairs(k, q, do, rate, n, reverse=True)
                if c["state"]:
                    ds = wide["dstate_out"][b, h]
                    dq += since * (do @ s0.T)
                    dk += left * (v @ ds.T)
                    dv += left * (k @ ds)
                    out["dstate_in"][b, h] = math.exp(-rate * n) * ds + scale * (since * q).T @ do
                out["dq"][at], out["dk"][at], out["dv"][at] = scale * dq, dk, dv
    return out


def _exact_norm_parts(t, kind, weight, bias):
    """The normalised values, their scale and the result."""
    if kind == "none":
        return None, None, t
    centred = t - t.mean(2, keepdim=True) if kind == "layer" else t
    r = 1.0 / torch.sqrt((centred ** 2).mean(2, keepdim=True) + EPS)
    unit = centred * r
    return unit, r, unit * weight + (0.0 if bias is None else bias)


def _exact_norm_back(dout, unit, r, kind, weight):
    """Gradients of a norm's input, weight and bias."""
    if kind == "none":
        return dout, None, None
    w = dout * weight
    inner = w - unit * (w * unit).mean(2, keepdim=True)
    if kind == "layer":
        inner = inner - w.mean(2, keepdim=True)
    return r * inner, (dout * unit).sum((0, 1)), dout.sum((0, 1))


def _exact_norm(c, s):
    names = ("x", "y", "gate_in", "pre_weight", "pre_bias", "post_weight", "post_bias", "dx_out", "dh")
    w = {n: None if s.get(n) is None else s[n].detach().double() for n in names}
    post_unit, post_r, u = _exact_norm_parts(w["y"], c["post"], w["post_weight"], w["post_bias"])
    if c["gate"] == "none":
        a = slope = None
        gated = u
    else:
        g = w["gate_in"]
        sig = 1.0 / (1.0 + torch.exp(-g))
        a, slope = {"none": (g, torch.ones_like(g)), "sigmoid": (sig, sig * (1 - sig)),
                    "silu": (g * sig, sig * (1 + g * (1 - sig)))}[c["act"]]
        gated = u * a
    x = w["x"] + c["alpha"] * gated
    pre_unit, pre_r, h = _exact_norm_parts(x, c["pre"], w["pre_weight"], w["pre_bias"])
    out = {"x": x}
    if c["pre"] != "none":
        out["h"] = h
    if c["op"] == "norm":
        return out
    dx, dpre_w, dpre_b = w["dx_out"], None, None
    if c["pre"] != "none":
        back, dpre_w, dpre_b = _exact_norm_back(w["dh"], pre_unit, pre_r, c["pre"], w["pre_weight"])
        dx = dx + back
    branch = c["alpha"] * dx
    dgate = None
    if c["gate"] != "none":
        dgate = branch * u * slope
        if c["gate"] != "token":
            dgate = dgate.sum(1, keepdim=True)
            if c["gate"] == "channel":
                dgate = dgate.sum((0, 1))
        branch = branch * a
    dy, dpost_w, dpost_b = _exact_norm_back(branch, post_unit, post_r, c["post"], w["post_weight"])
    grads = dict(x=dx, y=dy, gate_in=dgate, pre_weight=dpre_w, pre_bias=dpre_b, post_weight=dpost_w, post_bias=dpost_b)
    for name in _norm_leaves(s):
        out["d" + name] = grads[name]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return (_exact_norm if case["op"].startswith("norm") else _exact_decay)(case, s)
