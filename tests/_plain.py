"""Plain implementations, in 64 bits on the CPU, of the decay mixer and the residual norm: token by token and row by row from
their formulas, with the gradients written out.  Shared by the tests; nothing of the package is used."""
import torch


def decay(q, k, v, log_decay, scale, lengths=None, state=None):
    """q, k, v [B,H,N,d] fp64 -> o, state_out; tokens behind an item's length give zeros and leave the state."""
    B, H, N, d = q.shape
    s = torch.zeros(B, H, d, d, dtype=q.dtype) if state is None else state
    fade = log_decay.to(q.dtype).exp().view(1, H, 1, 1)
    outs = []
    for t in range(N):
        new = fade * s + k[:, :, t].unsqueeze(3) * v[:, :, t].unsqueeze(2)
        live = torch.ones(B, dtype=torch.bool) if lengths is None else lengths > t
        live = live.view(B, 1, 1, 1)
        s = torch.where(live, new, s)
        o = scale * (q[:, :, t].unsqueeze(3) * s).sum(2)
        outs.append(torch.where(live[..., 0], o, torch.zeros_like(o)))
    return torch.stack(outs, 2), s


def decay_gradients(q, k, v, log_decay, d_o, scale, lengths=None, state=None, dstate_out=None):
    """dq, dk, dv, dstate_in by the backward recurrence."""
    B, H, N, d = q.shape
    fade = log_decay.to(q.dtype).exp().view(1, H, 1, 1)
    g = torch.zeros(B, H, d, d, dtype=q.dtype) if dstate_out is None else dstate_out
    s = torch.zeros(B, H, d, d, dtype=q.dtype) if state is None else state
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    lives = [(torch.ones(B, dtype=torch.bool) if lengths is None else lengths > t).view(B, 1, 1, 1) for t in range(N)]
    for t in range(N):
        s = torch.where(lives[t], fade * s + k[:, :, t].unsqueeze(3) * v[:, :, t].unsqueeze(2), s)
        dq[:, :, t] = torch.where(lives[t][..., 0], scale * (s * d_o[:, :, t].unsqueeze(2)).sum(3), torch.zeros_like(dq[:, :, t]))
    for t in reversed(range(N)):
        ds = scale * q[:, :, t].unsqueeze(3) * d_o[:, :, t].unsqueeze(2) + g
        live = lives[t]
        dk[:, :, t] = torch.where(live[..., 0], (ds * v[:, :, t].unsqueeze(2)).sum(3), dk[:, :, t])
        dv[:, :, t] = torch.where(live[..., 0], (ds * k[:, :, t].unsqueeze(3)).sum(2), dv[:, :, t])
        g = torch.where(live, fade * ds, g)
    return dq, dk, dv, g


def _one_norm(t, kind, weight, bias, eps):
    if kind == "none":
        return t, None, t
    c = t - t.mean(1, keepdim=True) if kind == "layer" else t
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    unit = c * r
    out = unit if weight is None else unit * weight
    return unit, r, out if bias is None else out + bias


def act(g, kind):
    """Value and slope of what a gate goes through."""
    s = 1 / (1 + torch.exp(-g))
    return {"none": (g, torch.ones_like(g)), "sigmoid": (s, s * (1 - s)), "silu": (g * s, s * (1 + g * (1 - s)))}[kind]


def residual_norm(x, y, gate, p, pre, post, gate_act, alpha, eps):
    """x, y [rows,C], gate [rows,C] (already repeated) or None, p: dict of weights -> x_out, h and what the gradients need."""
    uh, r_post, u = _one_norm(y, post, p.get("post_weight"), p.get("post_bias"), eps) if y is not None else (None, None, None)
    a = u if gate is None else u * act(gate, gate_act)[0]
    x_out = x if y is None else x + alpha * a
    xh, r_pre, h = _one_norm(x_out, pre, p.get("pre_weight"), p.get("pre_bias"), eps)
    return x_out, (None if pre == "none" else h), dict(u=u, uh=uh, r_post=r_post, xh=xh, r_pre=r_pre)


def _norm_back(d, unit, r, kind, weight):
    if kind == "none":
        return d
    w = d if weight is None else d * weight
    m0 = w.mean(1, keepdim=True) if kind == "layer" else 0
    return r * (w - m0 - unit * (w * unit).mean(1, keepdim=True))


def residual_norm_gradients(x, y, gate, p, pre, post, gate_act, alpha, eps, dx_out, dh):
    """Gradients by name (the gate's per row; dx_out and dh zero where None)."""
    _, _, s = residual_norm(x, y, gate, p, pre, post, gate_act, alpha, eps)
    out = {}
    gx = torch.zeros_like(x) if dx_out is None else dx_out
    if pre != "none" and dh is not None:
        gx = gx + _norm_back(dh, s["xh"], s["r_pre"], pre, p.get("pre_weight"))
        out["pre_weight"], out["pre_bias"] = (dh * s["xh"]).sum(0), dh.sum(0)
    out["x"] = gx
    if y is not None:
        d = alpha * gx
        if gate is not None:
            value, slope = act(gate, gate_act)
            out["gate"] = d * s["u"] * slope
            d = d * value
        if post != "none":
            out["post_weight"], out["post_bias"] = (d * s["uh"]).sum(0), d.sum(0)
        out["y"] = _norm_back(d, s["uh"], s["r_post"], post, p.get("post_weight"))
    return out
