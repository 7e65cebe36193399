"""The decay mixer's outputs over its inputs: the buffers that may be one."""
import pytest
import torch

from paper_2508_12594_amd import binding
from tests.test_gpu_decay import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,d,dtype", [(1, 1, 128, "bf16"), (5, 7, 64, "f32"), (60, 8, 128, "f16"), (9, 3, 32, "bf16"),
                                         (300, 2, 64, "bf16")])
def test_step_writes_over_its_inputs(B, H, d, dtype):
    """With few (b,h) several workgroups share a state: none may write o before the others have read q and k."""
    print("[case] step over its inputs B%d H%d d%d %s" % (B, H, d, dtype), flush=True)
    dev, _ = make(B, H, 1, d, dtype, 41, state=True)
    tok = [dev[n][:, :, 0].contiguous() for n in ("q", "k", "v")]
    want_state = torch.empty_like(dev["state"])
    want = binding.decay_step(*tok, dev["log_decay"], dev["state"], 0.25, state_out=want_state)
    tol = (2 * d + 4) * 2.0 ** -24          # sums of d terms in another order
    size = 0.25 * (tok[0].double().abs().unsqueeze(3) * want_state.double().abs()).sum(2)
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]
    for i in range(3):
        mine = [t.clone() for t in tok]
        state = dev["state"].clone()
        o = binding.decay_step(*mine, dev["log_decay"], state, 0.25, o=mine[i])
        assert o is mine[i] and torch.equal(state, want_state), "qkv"[i]
        # (two roundings that may go different ways, by a half step each)
        assert ((o.double() - want.double()).abs() <= tol * size + 2 * u * want.double().abs() + 2.0 ** -24).all(), "qkv"[i]


@pytest.mark.parametrize("d,dtype,N,layout", [(128, "bf16", 1500, "bnhd"), (32, "f32", 200, "bhnd")])
def test_sequences_write_over_their_inputs(d, dtype, N, layout):
    """o over k and over v too, the state over the one that came in; a buffer that only begins at the same place is refused."""
    print("[case] sequences over their inputs d%d %s N%d %s" % (d, dtype, N, layout), flush=True)
    dev, _ = make(1, 3, N, d, dtype, 47, layout, state=True)
    names = ("q", "k", "v")
    want, want_state = binding.decay_forward(*(dev[n] for n in names), dev["log_decay"], 0.2, state=dev["state"], want_state=True,
                                             layout=layout)
    for i in range(3):
        mine, state = [dev[n].clone() for n in names], dev["state"].clone()
        o, _ = binding.decay_forward(*mine, dev["log_decay"], 0.2, state=state, state_out=state, o=mine[i], layout=layout)
        assert o is mine[i] and torch.equal(o, want) and torch.equal(state, want_state), names[i]
    room = torch.empty(dev["q"].numel() + 64, dtype=dev["q"].dtype, device="cuda")
    q, shifted = room[:-64].view_as(dev["q"]), room[64:].view_as(dev["q"])
    with pytest.raises(binding.FlareError):
        binding.decay_forward(q, dev["k"], dev["v"], dev["log_decay"], 0.2, o=shifted, layout=layout)
