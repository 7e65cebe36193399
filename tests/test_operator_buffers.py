"""Buffers that may not be one, refused on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2508_12594_amd import binding
from paper_2508_12594_amd.binding import DecayShape, NormParams, NormShape

ONE = ctypes.c_float(1)
X, Y, O, H = (ctypes.c_void_p(i << 24) for i in range(1, 5))      # never dereferenced, and far from each other


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_an_fp32_stream_does_not_fit_16_bit_buffers(lib):
    """Beside 16-bit branches the rows of an fp32 residual stream are twice as long: neither may lie in the other's buffer."""
    shape = ctypes.byref(NormShape(10, 64, binding.FLARE_BF16, 1, 1, 0, 0, 1))
    fwd = lib.flare_residual_norm_forward
    assert fwd(shape, None, X, Y, None, Y, H, None, ONE, ONE, None) == -1          # x_out over y
    assert fwd(shape, None, X, Y, None, O, X, None, ONE, ONE, None) == -1          # h over x
    assert fwd(shape, None, X, None, None, None, X, None, ONE, ONE, None) == -1


def test_decay_buffers(lib):
    """Every output over every input that it may not share, over the other outputs, and partly over what it may."""
    at = lambda i, off=0: ctypes.c_void_p((i << 24) + off)      # noqa: E731
    shape = DecayShape(2, 3, 100, 64, binding.FLARE_BF16, 0)
    rows, states = 2 * 3 * 100 * 64 * 2, 2 * 3 * 64 * 64 * 4
    good = [at(i) for i in range(1, 10)]                         # q, k, v, log_decay, lengths, state, o, state_out, marks

    def refused(call, args, i, p):
        return call(*args[:i], p, *args[i + 1:]) == -1

    forward = lambda *a: lib.flare_decay_forward(ctypes.byref(shape), *a, ONE, None, 0, None)    # noqa: E731
    long = DecayShape(1, 1, 5000, 64, binding.FLARE_BF16, 0)
    f, b, m = (ctypes.c_size_t(0) for _ in range(3))
    lib.flare_decay_workspace_bytes(ctypes.byref(long), 1, ctypes.byref(f), ctypes.byref(b), ctypes.byref(m))
    assert f.value and m.value
    for ws, marks in ((9, None), (None, 9)):                     # what is written on the way over an input
        for over in range(1, 9):
            a = good[:8] + [None]
            a[8] = at(over) if marks else None
            assert lib.flare_decay_forward(ctypes.byref(long), *a, ONE, at(over) if ws else None, f.value, None) == -1
    for i, allowed in ((6, (0, 1, 2)), (7, (5,))):
        for j in range(9):
            if j != i and j not in allowed and j != 8:           # (no marks: this shape is one segment)
                assert refused(forward, good, i, good[j]), (i, j)
            if j in allowed:                                     # not quite the same buffer, from either side
                size = rows if i == 6 else states
                assert refused(forward, good, i, at(j + 1, 16)) and refused(forward, good, i, at(j + 1, size - 16)), (i, j)
                assert refused(forward, good, i, at(j + 1, 16 - size)), (i, j)

    back = [at(i) for i in range(1, 14)]      # q, k, v, log_decay, lengths, state, marks, d_o, dstate_out, dq, dk, dv, dstate
    backward = lambda *a: lib.flare_decay_backward(ctypes.byref(shape), *a, ONE, None, 0, None)   # noqa: E731
    for i in range(9, 13):
        for j in range(13):
            if j != i and j != 6:
                assert refused(backward, back, i, back[j]), (i, j)
        assert refused(backward, back, i, at(1, rows - 16))

    token = DecayShape(2, 3, 1, 64, binding.FLARE_BF16, 0)
    step = lambda *a: lib.flare_decay_step(ctypes.byref(token), *a, ONE, None)    # noqa: E731
    args = [at(i) for i in range(1, 9)]                          # q, k, v, log_decay, active, state, state_out, o
    for i, allowed in ((6, (5,)), (7, (0, 1, 2))):
        for j in range(8):
            if j != i and j not in allowed:
                assert refused(step, args, i, args[j]), (i, j)
            if j in allowed:
                assert refused(step, args, i, at(j + 1, 16)), (i, j)


def test_norm_buffers(lib):
    at = lambda i, off=0: ctypes.c_void_p((i << 24) + off)      # noqa: E731
    params = NormParams(*(at(i) for i in (20, 21, 22, 23)))
    shape = NormShape(10, 64, binding.FLARE_BF16, 0, 1, 2, 2, 5)
    forward = lambda *a: lib.flare_residual_norm_forward(ctypes.byref(shape), ctypes.byref(params), *a, ONE, ONE, None)   # noqa: E731
    args = [at(i) for i in range(1, 7)]                          # x, y, gate, x_out, h, stats
    for i, over in ((3, (3, 5, 6, 20, 21, 22, 23)), (4, (3, 4, 6, 20, 23)), (5, (1, 2, 3, 4, 5, 21))):
        for j in over:
            assert forward(*args[:i], at(j), *args[i + 1:]) == -1, (i, j)
    for i, j in ((3, 1), (3, 2), (4, 1), (4, 2)):
        assert forward(*args[:i], at(j, 128), *args[i + 1:]) == -1, (i, j)

    size = ctypes.c_size_t(0)
    assert lib.flare_residual_norm_workspace_bytes(ctypes.byref(shape), ctypes.byref(size)) == 0
    back = [at(i) for i in range(1, 14)]      # x, y, gate, stats, dx_out, dh, dx, dy, dgate, and the four of the params

    def backward(a, ws=at(14), s=shape):
        return lib.flare_residual_norm_backward(ctypes.byref(s), ctypes.byref(params), *a, ONE, ws, size, None)

    for i in range(6, 13):
        may = {6: (0, 1, 4, 5), 7: (0, 1, 4, 5)}.get(i, ())
        for j in list(range(13)) + [19, 20, 21, 22]:
            if j != i and j not in may:
                assert backward(back[:i] + [at(j + 1)] + back[i + 1:]) == -1, (i, j)
            if j in may:
                assert backward(back[:i] + [at(j + 1, 16)] + back[i + 1:]) == -1, (i, j)
        assert backward(back, ws=back[i]) == -1
    for i in range(6):
        assert backward(back, ws=back[i]) == -1
    wide = NormShape(10, 64, binding.FLARE_BF16, 1, 1, 2, 2, 5)  # an fp32 stream: other rows
    for i, j in ((6, 1), (6, 5), (7, 0), (7, 4)):
        assert backward(back[:i] + [back[j]] + back[i + 1:], s=wide) == -1, (i, j)
