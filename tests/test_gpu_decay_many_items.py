"""Padded batches of very many items, each in one segment."""
import pytest
import torch

from paper_2508_12594_amd import binding
from tests import _plain
from tests.test_gpu_decay import check, magnitudes, make

pytestmark = pytest.mark.gpu


def test_as_many_items_as_there_may_be():
    """65535 sequences of 0 to 33 tokens: no workgroup may search the batch for its item.  A sample of them is compared."""
    B, N, d = 65535, 33, 16
    lengths = [(11 * b) % (N + 1) for b in range(B)]
    print("[case] %d items" % B, flush=True)
    dev, wide = make(B, 1, N, d, "bf16", 51, lengths=lengths, decays=[-0.03])
    args = [dev[n] for n in ("q", "k", "v", "log_decay")]
    o, s = binding.decay_forward(*args, 0.25, lengths=dev["lengths"], want_state=True)
    grads = binding.decay_backward(*args, dev["d_o"], 0.25, lengths=dev["lengths"])[:3]
    some = torch.arange(0, B, 331)
    part = {n: a if n == "log_decay" or a is None else a[some] for n, a in wide.items()}
    names = ("q", "k", "v", "log_decay")
    want, size = (_plain.decay(*(w[n] for n in names), 0.25, w["lengths"]) for w in (part, magnitudes(part)))
    wgrad, gsize = (_plain.decay_gradients(*(w[n] for n in names), w["d_o"], 0.25, w["lengths"]) for w in (part, magnitudes(part)))
    for name, got, exact, mag in zip(("o", "dq", "dk", "dv"), (o,) + grads, want[:1] + wgrad[:3], size[:1] + gsize[:3]):
        check(name, got.cpu()[some].double(), exact, mag, "bf16", N, d, 2)
    check("state", s.cpu()[some].double(), want[1], size[1], "f32", N, d, 1)
    live = torch.arange(N) < torch.tensor(lengths).unsqueeze(1)
    for t in (o,) + grads:
        assert (t.cpu()[~live.view(B, 1, N)] == 0).all()
