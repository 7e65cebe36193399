"""What the decay mixer and the residual norm refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.binding import DecayShape, FlareError, NormParams, NormShape

P, ODD, ONE = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_float(1)   # never dereferenced: the checks fail first
A, B, C, S, T = (ctypes.c_void_p(4096 * i) for i in range(2, 7))                # other buffers


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_decay_shapes(lib):
    good = (2, 3, 100, 64, binding.FLARE_BF16, 0)
    f, b = ctypes.c_size_t(1), ctypes.c_size_t(1)
    assert lib.flare_decay_workspace_bytes(ctypes.byref(DecayShape(*good)), 0, ctypes.byref(f), ctypes.byref(b), None) == 0
    assert lib.flare_decay_workspace_bytes(None, 0, None, None, None) == -1
    bad = [(0, 3, 100, 64, 1, 0, -1), (2, 0, 100, 64, 1, 0, -1), (2, 3, 0, 64, 1, 0, -1), (2, 3, 100, 0, 1, 0, -1),
           (2, 3, 100, 48, 1, 0, -2), (2, 3, 100, 256, 1, 0, -2), (2, 3, 100, 8, 1, 0, -2), (2, 3, 100, 64, 3, 0, -2),
           (2, 3, 100, 64, 1, 2, -2), (70000, 1, 100, 64, 1, 0, -2), (1, 1, 1 << 24, 16, 1, 0, -2), (1, 300, 1 << 20, 128, 1, 1, -2)]
    for *shape, code in bad:
        assert lib.flare_decay_workspace_bytes(ctypes.byref(DecayShape(*shape)), 0, None, None, None) == code, shape


def test_decay_arguments(lib):
    one = ctypes.byref(DecayShape(1, 2, 40, 64, binding.FLARE_F16, 0))
    args = [P, P, P, P, None, None, P, None, None]
    for i in (0, 1, 2, 3, 6):
        a = list(args)
        a[i] = None
        assert lib.flare_decay_forward(one, *a, ONE, None, 0, None) == -1
    for i in range(9):
        a = list(args)
        a[i] = ODD
        assert lib.flare_decay_forward(one, *a, ONE, None, 0, None) == -3
    back = [P, P, P, P, None, None, None, P, None, A, B, C, None]
    for i in (0, 1, 2, 3, 7, 9, 10, 11):
        a = list(back)
        a[i] = None
        assert lib.flare_decay_backward(one, *a, ONE, None, 0, None) == -1
    for i in range(13):
        a = list(back)
        a[i] = ODD
        assert lib.flare_decay_backward(one, *a, ONE, None, 0, None) == -3
    for i, other in ((9, P), (10, P), (11, P), (9, B), (10, C), (11, A)):          # an output over an input, over another output
        a = list(back)
        a[i] = other
        assert lib.flare_decay_backward(one, *a, ONE, None, 0, None) == -1
    for states in ((S, T, S), (T, S, S)):
        a = list(back)
        a[5], a[8], a[12] = states
        assert lib.flare_decay_backward(one, *a, ONE, None, 0, None) == -1
    # a long sequence of few heads is split, and needs its slots
    long = DecayShape(1, 1, 100000, 128, binding.FLARE_BF16, 0)
    f, b, m = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.flare_decay_workspace_bytes(ctypes.byref(long), 0, ctypes.byref(f), ctypes.byref(b), ctypes.byref(m)) == 0
    assert f.value and b.value and m.value
    assert lib.flare_decay_forward(ctypes.byref(long), *args, ONE, None, 0, None) == -4
    assert lib.flare_decay_forward(ctypes.byref(long), *args, ONE, P, f.value - 1, None) == -4
    assert lib.flare_decay_forward(ctypes.byref(long), *args, ONE, ODD, f.value, None) == -3
    assert lib.flare_decay_backward(ctypes.byref(long), *back, ONE, P, b.value - 1, None) == -4
    step = [P, P, P, P, None, P, P, P]
    token = ctypes.byref(DecayShape(1, 2, 1, 64, binding.FLARE_F16, 0))
    assert lib.flare_decay_step(one, *step, ONE, None) == -1                       # N is not 1
    for i in (0, 1, 2, 3, 5, 6, 7):
        a = list(step)
        a[i] = None
        assert lib.flare_decay_step(token, *a, ONE, None) == -1
        a[i] = ODD
        assert lib.flare_decay_step(token, *a, ONE, None) == -3


def norm_shape(rows=10, C=64, dtype=1, x_f32=0, pre=1, post=0, gate=0, rows_per_gate=1):
    return ctypes.byref(NormShape(rows, C, dtype, x_f32, pre, post, gate, rows_per_gate))


def test_norm_shapes(lib):
    size = ctypes.c_size_t(0)
    assert lib.flare_residual_norm_workspace_bytes(norm_shape(), ctypes.byref(size)) == 0 and size.value > 0
    assert lib.flare_residual_norm_workspace_bytes(None, ctypes.byref(size)) == -1
    for code, over in [(-1, dict(rows=0)), (-1, dict(C=0)), (-2, dict(C=8193)), (-2, dict(rows=1 << 31)), (-2, dict(dtype=5)),
                       (-1, dict(x_f32=2)), (-1, dict(pre=3)), (-1, dict(post=-1)), (-1, dict(gate=4)),
                       (-1, dict(gate=1, rows_per_gate=3)), (-1, dict(gate=1, rows_per_gate=0))]:
        assert lib.flare_residual_norm_workspace_bytes(norm_shape(**over), ctypes.byref(size)) == code, over


def test_norm_arguments(lib):
    fwd = lib.flare_residual_norm_forward
    weights = NormParams(P, None, None, None)
    post = NormParams(None, None, None, P)
    crooked = NormParams(ODD, None, None, None)
    assert fwd(norm_shape(), None, None, P, None, P, P, None, ONE, ONE, None) == -1          # no x
    assert fwd(norm_shape(), None, P, None, None, P, P, None, ONE, ONE, None) == -1          # x_out without y
    assert fwd(norm_shape(), None, P, P, None, None, P, None, ONE, ONE, None) == -1          # y without x_out
    assert fwd(norm_shape(), None, P, P, None, P, None, None, ONE, ONE, None) == -1          # a pre norm without h
    assert fwd(norm_shape(pre=0), None, P, P, None, P, P, None, ONE, ONE, None) == -1        # h without a pre norm
    assert fwd(norm_shape(pre=0), None, P, None, None, None, None, None, ONE, ONE, None) == -1
    assert fwd(norm_shape(post=1), None, P, None, None, None, P, None, ONE, ONE, None) == -1  # a post norm of nothing
    assert fwd(norm_shape(gate=1), None, P, P, None, P, P, None, ONE, ONE, None) == -1       # no gate
    assert fwd(norm_shape(), None, P, P, P, P, P, None, ONE, ONE, None) == -1                # a gate that is none
    assert fwd(norm_shape(pre=0), ctypes.byref(weights), P, P, None, P, None, None, ONE, ONE, None) == -1
    assert fwd(norm_shape(), ctypes.byref(post), P, P, None, P, P, None, ONE, ONE, None) == -1
    assert fwd(norm_shape(), ctypes.byref(crooked), P, P, None, P, P, None, ONE, ONE, None) == -3
    assert fwd(norm_shape(), None, P, P, None, A, A, None, ONE, ONE, None) == -1                # two outputs in one buffer
    for i in (0, 1, 3, 4, 5):
        a = [P, P, None, A, B, P]
        a[i] = ODD
        assert fwd(norm_shape(), None, *a, ONE, ONE, None) == -3
    bwd = lib.flare_residual_norm_backward

    def call(shape, x=P, y=P, gate=None, stats=P, dx_out=P, dh=P, dx=P, dy=A, dgate=None, w=(None,) * 4, ws=P, size=1 << 30):
        return bwd(shape, None, x, y, gate, stats, dx_out, dh, dx, dy, dgate, *w, ONE, ws, size, None)

    assert call(norm_shape(), x=None) == -1 and call(norm_shape(), stats=None) == -1
    assert call(norm_shape(), y=None) == -1                                                 # gradients of what is not there
    assert call(norm_shape(), dgate=P) == -1 and call(norm_shape(), w=(None, None, P, None)) == -1
    assert call(norm_shape(pre=0), dh=P) == -1 and call(norm_shape(pre=0), dh=None, w=(P, None, None, None)) == -1
    assert call(norm_shape(), dy=P) == -1 and call(norm_shape(gate=1), gate=B, dgate=A) == -1
    assert call(norm_shape(gate=1), gate=B, dgate=B) == -1
    assert call(norm_shape(), ws=None) == -4 and call(norm_shape(), size=16) == -4
    assert call(norm_shape(), ws=ODD) == -3 and call(norm_shape(), dy=ODD) == -3 and call(norm_shape(), w=(ODD, None, None, None)) == -3


def test_tensors_on_the_host_and_names(lib):
    """Through the Python entry points: host tensors and unknown names are errors of the package."""
    from paper_2508_12594_amd.autograd import decay_mixer, residual_norm
    q, g = torch.zeros(1, 2, 4, 16), torch.zeros(2)
    for call in (lambda: binding.decay_forward(q, q, q, g, 1.0), lambda: decay_mixer(q, q, q, g, 1.0),
                 lambda: binding.decay_backward(q, q, q, g, q, 1.0), lambda: binding.decay_forward(q, q, q, g, 1.0, layout="nhd"),
                 lambda: binding.decay_step(q[:, :, 0], q[:, :, 0], q[:, :, 0], g, torch.zeros(1, 2, 16, 16), 1.0),
                 lambda: binding.residual_norm_forward(q, q), lambda: residual_norm(q, q),
                 lambda: binding.residual_norm_backward(q, q, q, q, g), lambda: residual_norm(q, q, pre="batch"),
                 lambda: residual_norm(q, q, q, gate_act="tanh")):
        with pytest.raises(FlareError):
            call()
