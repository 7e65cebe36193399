"""The residual norm's outputs over its inputs: every pair that the header allows."""
import ctypes

import pytest
import torch

from paper_2508_12594_amd import binding
from tests.test_gpu_residual_norm import PARAMS, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype,x_f32", [((70, 64), "bf16", False), ((9, 8192), "f16", False), ((301, 250), "f32", False),
                                               ((40, 512), "bf16", True), ((5, 2049), "f16", True)])
def test_forward_over_its_inputs(shape, dtype, x_f32):
    print("[case] norm over its inputs %s %s x_f32=%s" % (shape, dtype, x_f32), flush=True)
    t = {n: None if a is None else a.cuda() for n, a in make(shape, dtype, x_f32, "layer", "rms", "token", True, True, 3).items()}
    given = dict({n: t[n] for n in PARAMS}, pre="layer", post="rms", gate_act="silu")
    want = binding.residual_norm_forward(t["x"], t["y"], t["gate"], **given)
    pairs = [("x", "y"), ("x", None), (None, "y")] + ([] if x_f32 else [("y", "x"), ("y", None), (None, "x")])
    for over_x, over_h in pairs:
        mine = {n: t[n].clone() for n in ("x", "y")}
        got = binding.residual_norm_forward(mine["x"], mine["y"], t["gate"], x_out=mine.get(over_x), h=mine.get(over_h), **given)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (over_x, over_h)


@pytest.mark.parametrize("shape,dtype,x_f32", [((70, 64), "bf16", False), ((9, 8192), "f16", False), ((301, 250), "f32", False),
                                               ((40, 512), "bf16", True), ((5, 2049), "f16", True)])
def test_backward_over_its_inputs(shape, dtype, x_f32):
    print("[case] norm gradients over the inputs %s %s x_f32=%s" % (shape, dtype, x_f32), flush=True)
    lib = binding.load()
    t = {n: None if a is None else a.cuda() for n, a in make(shape, dtype, x_f32, "layer", "rms", "none", False, False, 5).items()}
    stats = torch.empty(shape[0], 4, device="cuda")
    binding.residual_norm_forward(t["x"], t["y"], pre="layer", post="rms", stats=stats)
    want = binding.residual_norm_backward(t["x"], t["y"], t["dx_out"], t["dh"], stats, pre="layer", post="rms")[:2]
    s = binding.NormShape(shape[0], shape[1], binding._dtype_code(t["y"]), int(x_f32), 1, 2, 0, 1)
    size = ctypes.c_size_t(0)
    assert lib.flare_residual_norm_workspace_bytes(ctypes.byref(s), ctypes.byref(size)) == 0
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    names = ("x", "y", "dx_out", "dh")
    free = {"dx": torch.empty_like(t["x"]), "dy": torch.empty_like(t["y"])}
    for over_dx in ("x", "dx_out", None) if x_f32 else names + (None,):
        for over_dy in ("y", "dh", None) if x_f32 else names + (None,):
            if over_dx == over_dy:
                continue
            mine = {n: t[n].clone() for n in names}
            dx, dy = mine.get(over_dx, free["dx"]), mine.get(over_dy, free["dy"])
            p = lambda a: ctypes.c_void_p(a.data_ptr())      # noqa: E731
            rc = lib.flare_residual_norm_backward(
                ctypes.byref(s), None, p(mine["x"]), p(mine["y"]), None, p(stats), p(mine["dx_out"]), p(mine["dh"]), p(dx), p(dy),
                None, None, None, None, None, ctypes.c_float(1), p(ws), size,
                ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
            assert rc == 0 and torch.equal(dx, want[0]) and torch.equal(dy, want[1]), (over_dx, over_dy)
