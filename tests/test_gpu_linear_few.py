"""Products on few pixels, where a wave's steps of k go out several at once or one after the other: the
same sums in the same order, at sizes on both sides of each of the rule's limits."""
import pytest
import torch

import act_ref as A
import block_ref as R
import paper_1903_06681_amd as dc
import test_gpu_act as T
import test_gpu_block_ops as B

pytestmark = pytest.mark.gpu
V = dc.View.of
_gpu = T._gpu

# pixels (one, two, three tiles of 16), channels for one to five steps of k a wave, whole and not; many workgroups
PIXELS = {"rows": [(7, 1, 1), (24, 1, 1), (50, 1, 1)], "dense": [(1, 2, 3), (1, 4, 6), (2, 5, 5)]}
CHANNELS = [96, 511, 530, 800, 1024, 1030, 1290]
SIZES = [(layout, p, C, K) for layout, some in PIXELS.items() for p in some for C, K in [(c, 40) for c in CHANNELS] + [(530, 4130), (1024, 2070)]]


@pytest.mark.parametrize("layout,pixels,C,K", SIZES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_on_few_pixels(layout, pixels, C, K, dtype):
    """Within the bounds of C products and the bias in fp32, both ways (the slope's and the activation's own
    errors as for the gated product: 1.13 of the sum's, 1e-6 and 4e-7)."""
    N, H, W = pixels
    g = T.rng(31)
    x, _ = T.put(layout, T.randn(g, N, C, H, W), dtype)
    w, b = (T.randn(g, K, C) / C ** 0.5).to(A.DT[dtype]).cuda(), B.vec(g, K)
    (y, mem), (z, zmem) = A.tensor(layout, N, K, H, W, "f32"), A.tensor(layout, N, K, H, W, "f32")
    dc.linear_fwd(V(x), x, w, b, dc.DC_ACT_GELU, None, None, V(z), z, V(y), y)
    want = R.product(w.double(), B.f64(x)) + b.double()[:, None]
    e = (C + 2) * R.EPS32 * (R.product(w.double().abs(), B.f64(x).abs()) + b.double().abs()[:, None])
    B.near(z, want, e, "z")
    B.near(y, R.act(want, "gelu"), 1.13 * e + 4e-7 * want.abs() + R.EPS32 * want.abs(), "y")
    assert A.untouched(y, mem) and A.untouched(z, zmem)
    w2 = (T.randn(g, C, K) / C ** 0.5).to(A.DT[dtype]).cuda()
    dx, dmem = A.tensor(layout, N, K, H, W, "f32")
    dc.linear_bwd_data(V(x), x, w2, dc.DC_ACT_GELU, V(z), z, None, None, V(dx), dx)
    p = R.product(w2.double().t().contiguous(), B.f64(x))
    ep = (C + 2) * R.EPS32 * R.product(w2.double().abs().t().contiguous(), B.f64(x).abs())
    B.near(dx, p * R.slope(B.f64(z), "gelu"), 1.13 * ep + 1e-6 * p.abs() + 2 * R.EPS32 * p.abs(), "dx")
    assert A.untouched(dx, dmem)
