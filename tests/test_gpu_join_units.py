"""Backward pass of the join where the gates' units (slices of a sample's pixels, each taken by one
workgroup) do not fill the last turn of the workgroups: those without a unit leave the sums of
the others alone.  A size for every form of the kernel; test_join_plan.py checks that it is one."""
import pytest
import torch

import block_ref as R
import paper_1903_06681_amd as dc
import test_gpu_act as T
import test_gpu_block_ops as B

pytestmark = pytest.mark.gpu
V = dc.View.of
_gpu = T._gpu

# (pixels a wave, eights a lane; 0: one by one, any number), rows of channels or planes
UNITS = {
    ("rows", 16, 1): [(1030, 20, 1, 1)],
    ("rows", 8, 1): [(1030, 60, 1, 1)],
    ("rows", 4, 1): [(1030, 120, 1, 1)],
    ("rows", 2, 1): [(1030, 250, 1, 1)],
    ("rows", 1, 1): [(37, 500, 17, 1)],
    ("rows", 1, 2): [(3, 5000, 100, 1)],
    ("rows", 1, 0): [(3, 8200, 100, 1), (300, 8200, 1, 1)],
    ("dense", 64, 1): [(515, 20, 1, 2)],
    ("dense", 16, 1): [(300, 200, 1, 2)],
    ("dense", 4, 1): [(515, 300, 1, 2)],
    ("dense", 4, 2): [(300, 1500, 1, 2)],
    ("dense", 16, 0): [(300, 2056, 1, 2), (3, 2056, 30, 50), (5, 2304, 64, 64)],
}
SIZES = [(s, form[0]) for form, sizes in UNITS.items() for s in sizes]


@pytest.mark.parametrize("shape,layout", SIZES, ids=str)
@pytest.mark.parametrize("name", ["all", "mixed"])
def test_units_that_do_not_fill_the_last_turn(shape, layout, name):
    """Values and bounds as for every other size; the workspace holds NaN before each call."""
    B.check_join(shape, layout, **B.JOINS[name])


@pytest.mark.parametrize("shape,layout", SIZES, ids=str)
def test_the_same_bits_from_call_to_call(shape, layout):
    """The order of summation is fixed, whatever the workspace holds before."""
    N, C, H, W = shape
    g = T.rng(21)
    y, x, du = (T.put(layout, T.randn(g, *shape), "f32")[0] for _ in range(3))
    scale, gate = B.vec(g, C, mean=0.5), B.vec(g, N, C, mean=1.0)
    post, pre, drop = dc.Norm(dc.DC_NORM_RMS, B.EPS), dc.Norm(dc.DC_NORM_LAYER, B.EPS), dc.Drop(0.2, 9)
    o, u, stat = torch.empty_like(x), torch.empty_like(x), torch.empty(4, N, H, W, device="cuda")
    dc.join_fwd(V(y), y, post, scale, gate, drop, V(x), x, pre, V(o), o, V(u), u, stat)
    found = []
    for fill in (0, 255, 255):
        grads = dc.JoinGrads(*(torch.full(s, float("nan"), device="cuda") for s in ((C,), (N, C), (C,), (C,), (C,), (C,))))
        dx, dy, mem = torch.empty_like(x), torch.empty_like(y), T.ws(dc.join_bwd_workspace_bytes(V(y), True)).fill_(fill)
        dc.join_bwd(V(du), du, None, None, V(y), y, V(x), x, None, None, stat, post, scale, gate, drop, pre, V(dx), dx, V(dy), dy, grads, 0, mem)
        found.append([dx, dy, grads.scale, grads.gate, grads.gamma_post, grads.beta_post, grads.gamma_pre, grads.beta_pre])
    for other in found[1:]:
        for a, b in zip(found[0], other):
            assert torch.equal(a, b)
    assert all(bool(torch.isfinite(t).all()) for t in found[0])
    # a gate's gradient times the gate, over the samples, is the scale's times the scale: two sums of the same terms,
    # a pixel each, in fp32
    s, k = found[0][2].double() * scale.double(), (found[0][3].double() * gate.double()).sum(0)
    size = (found[0][3].double() * gate.double()).abs().sum(0)
    assert bool(((s - k).abs() <= (N + 6) * R.EPS32 * size).all())
