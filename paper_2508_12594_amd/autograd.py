"""torch.autograd wrappers around the binding: `flare_mixer(q_lat, k, v, scale)`, `decay_mixer(q, k, v, log_decay, scale)`
and `residual_norm(x, y)` are differentiable.

Nothing is computed here: the forward calls flare_forward (keeping z, lse_enc, lse_dec and y for the
backward), the backward calls flare_backward_cast (dq_lat in q_lat's dtype, which autograd requires of a
gradient).  The autograd node is native (csrc/torch_binding.cpp, MixerBackward).  This is how the paper's layer
would use the operator in place of its two attention calls (listing in Section 3.1).
"""
from . import binding

_RECORDED = None


def _recorded():
    """The same step as a torch.autograd.Function, which torch.jit.trace records as an operation of the graph."""
    global _RECORDED
    if _RECORDED is None:
        import torch

        class RecordedMixer(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q_lat, k, v, scale, layout, y_f32):
                q_lat, k, v = q_lat.contiguous(), k.contiguous(), v.contiguous()
                B, H, N = k.shape[:3] if layout == "bhnd" else (k.shape[0], k.shape[2], k.shape[1])
                lse_dec = torch.empty((B, H, N), dtype=torch.float32, device=k.device)
                y, z, lse_enc = binding.forward(q_lat, k, v, scale, lse_dec=lse_dec, layout=layout, y_f32=y_f32)
                ctx.save_for_backward(q_lat, k, v, y, z, lse_enc, lse_dec)
                ctx.scale, ctx.layout = scale, layout
                return y

            @staticmethod
            def backward(ctx, dy):
                q_lat, k, v, y, z, lse_enc, lse_dec = ctx.saved_tensors
                dq, dk, dv = binding.backward(q_lat, k, v, dy.to(k.dtype).contiguous(), z, lse_enc, ctx.scale, y=y,
                                              lse_dec=lse_dec, layout=ctx.layout)
                return dq.to(q_lat.dtype), dk, dv, None, None, None

        _RECORDED = RecordedMixer
    return _RECORDED


def flare_mixer(q_lat, k, v, scale, layout="bhnd", y_f32=False):
    """y = FLARE(q_lat, k, v): q_lat [H,M,d] (or [M,d]: shared latents), k, v [B,H,N,d] ('bhnd') or
    [B,N,H,d] ('bnhd'); returns y in k's shape and dtype.  Differentiable in q_lat, k and v.

    y_f32 (16-bit inputs, at most 2048 latents): y comes back in fp32 and the backward reads it instead of
    recomputing the token statistics, which pays at d < 16 (flare_shape.y_f32)."""
    y = binding._native().mixer(q_lat, k, v, float(scale), binding._layout(layout), bool(y_f32))
    if y is None:
        y = _recorded().apply(q_lat, k, v, float(scale), layout, bool(y_f32))
    return y


_ONCE = None


def _once(of, grads, inputs):
    """Gradients that a graph is asked of are constants to it: a derivative of them, which would be lost without a word, raises."""
    import torch
    global _ONCE
    if not torch.is_grad_enabled():
        return grads
    if _ONCE is None:
        class Once(torch.autograd.Function):
            @staticmethod
            def forward(ctx, of, count, *tensors):
                ctx.of = of
                return tuple(t.view_as(t) for t in tensors[:count])

            @staticmethod
            def backward(ctx, *_):
                raise binding.FlareError(ctx.of + " has no second derivative")

        _ONCE = Once
    there = [g for g in grads if g is not None]
    made = iter(_ONCE.apply(of, len(there), *there, *(t for t in inputs if t is not None)))
    return tuple(None if g is None else next(made) for g in grads)


_RECORDED_DECAY = None


def _recorded_decay():
    global _RECORDED_DECAY
    if _RECORDED_DECAY is None:
        import torch

        class RecordedDecayMixer(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, v, log_decay, lengths, state, scale, want_state, layout):
                whole = lambda t: None if t is None else t.contiguous()   # noqa: E731
                q, k, v, log_decay, lengths, state = (whole(t) for t in (q, k, v, log_decay, lengths, state))
                o, state_out = binding.decay_forward(q, k, v, log_decay, scale, lengths=lengths, state=state,
                                                     want_state=want_state, layout=layout)
                ctx.save_for_backward(q, k, v, log_decay, lengths, state)
                ctx.scale, ctx.layout = scale, layout
                return (o, state_out) if want_state else o

            @staticmethod
            def backward(ctx, d_o, dstate_out=None):
                q, k, v, log_decay, lengths, state = ctx.saved_tensors
                dq, dk, dv, dstate = binding.decay_backward(
                    q, k, v, log_decay, d_o.contiguous(), ctx.scale, lengths=lengths, state=state,
                    dstate_out=None if dstate_out is None else dstate_out.contiguous(),
                    want_dstate=state is not None and ctx.needs_input_grad[5], layout=ctx.layout)
                dq, dk, dv, dstate = _once("decay_mixer", (dq, dk, dv, dstate), (q, k, v, state, d_o, dstate_out))
                return dq, dk, dv, None, None, dstate, None, None, None

        _RECORDED_DECAY = RecordedDecayMixer
    return _RECORDED_DECAY


def decay_mixer(q, k, v, log_decay, scale, lengths=None, state=None, want_state=False, layout="bhnd"):
    """Causal linear attention with a decay for each head (flare_decay_forward): per head S_t = exp(log_decay) S_{t-1} + k_t v_t^T,
    o_t = scale S_t^T q_t.  q, k, v [B,H,N,d] ('bhnd') or [B,N,H,d] ('bnhd'), log_decay [H] fp32 and at most 0 (a constant: it is
    not differentiated), lengths [B] int32 for a padded batch, state [B,H,d,d] fp32 from an earlier piece of the
    sequences.  Returns (o, state_out), state_out None without want_state.  Differentiable in q, k, v and state (once)."""
    out = binding._native().decay_mixer(q, k, v, log_decay, float(scale), lengths, state, bool(want_state),
                                        binding._layout(layout))
    if out is None:
        if log_decay.requires_grad:
            raise binding.FlareError("log_decay is not differentiated: pass it detached")
        out = _recorded_decay().apply(q, k, v, log_decay, lengths, state, float(scale), bool(want_state), layout)
        out = out if want_state else (out, None)
    return out


_RECORDED_NORM = None


def _recorded_norm():
    global _RECORDED_NORM
    if _RECORDED_NORM is None:
        import torch

        class RecordedResidualNorm(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, y, gate, pre_weight, pre_bias, post_weight, post_bias, kinds, eps, h_dtype):
                whole = lambda t: None if t is None else t.contiguous()   # noqa: E731
                tensors = [whole(t) for t in (x, y, gate, pre_weight, pre_bias, post_weight, post_bias)]
                stats = torch.empty((tensors[0].numel() // tensors[0].shape[-1], 4), dtype=torch.float32, device=x.device)
                names = ("pre_weight", "pre_bias", "post_weight", "post_bias")
                x_out, h = binding.residual_norm_forward(*tensors[:3], **dict(zip(names, tensors[3:])), **kinds, eps=eps,
                                                         stats=stats, h_dtype=h_dtype)
                ctx.save_for_backward(stats, *tensors)
                ctx.kinds, ctx.outputs = kinds, (x_out is not None, h is not None)
                return (x_out, h) if all(ctx.outputs) else h if x_out is None else x_out

            @staticmethod
            def backward(ctx, *grads):
                grads = [g if g is None else g.contiguous() for g in grads]
                dx_out = grads.pop(0) if ctx.outputs[0] else None
                dh = grads.pop(0) if ctx.outputs[1] else None
                stats, x, y, gate, *params = ctx.saved_tensors
                names = ("pre_weight", "pre_bias", "post_weight", "post_bias")
                out = binding.residual_norm_backward(x, y, dx_out, dh, stats, gate=gate, **dict(zip(names, params)), **ctx.kinds)
                return _once("residual_norm", out, [x, y, gate, dx_out, dh] + params) + (None, None, None)

        _RECORDED_NORM = RecordedResidualNorm
    return _RECORDED_NORM


def residual_norm(x, y=None, gate=None, pre="layer", post="none", pre_weight=None, pre_bias=None, post_weight=None, post_bias=None,
                  gate_act="none", alpha=1.0, eps=1e-5, h_dtype=None):
    """x_out = x + alpha * post(y) * gate_act(gate) and h = pre(x_out) in one pass (flare_residual_norm_forward; shapes as in
    binding.residual_norm_forward).  Returns (x_out, h): without y x_out is x, with pre 'none' h is None.  Differentiable in
    all tensors (once)."""
    kinds = dict(pre=pre, post=post, gate_act=gate_act, alpha=float(alpha))
    out = binding._native().residual_norm(x, y, gate, binding._norm(pre, "pre"), binding._norm(post, "post"), binding._gate(gate_act),
                                          pre_weight, pre_bias, post_weight, post_bias, float(alpha), float(eps), h_dtype)
    if out is None:
        made = _recorded_norm().apply(x, y, gate, pre_weight, pre_bias, post_weight, post_bias, kinds, float(eps), h_dtype)
        out = made if y is not None and pre != "none" else (None, made) if y is None else (made, None)
    return (x if y is None else out[0]), out[1]
