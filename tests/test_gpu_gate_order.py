"""The gated product's order of summation does not depend on where a pixel lies: the same channels in
another row of a batch, or another pixel of an image, give the same bits (as the plain product's),
forward and backward, in every block that the sizes pick."""
import pytest
import torch

import act_ref as A
import paper_1903_06681_amd as dc
import test_gpu_act as T
import test_gpu_block_ops as B

pytestmark = pytest.mark.gpu
V = dc.View.of
_gpu = T._gpu

# N, C, H, W, K: blocks of the sizes' largest to few pixels; sums of one slice, two, five and nine
SHAPES = {
    "large_rows": ((16, 512, 600, 1, 1024), "rows"), "large_rows_ragged": ((9000, 263, 1, 1, 1100), "slice"),
    "large": ((1, 136, 130, 300, 256), "dense"), "large_gaps": ((1, 330, 131, 133, 500), "gaps"),
    "middle": ((1, 128, 150, 304, 136), "dense"), "middle_rows": ((35, 128, 1000, 1, 136), "slice"),
    "short": ((2, 32, 200, 250, 72), "padded"), "small": ((2, 300, 30, 31, 130), "dense"), "small_rows": ((3, 520, 301, 1, 200), "rows"),
    "few": ((37, 520, 1, 1, 140), "rows"),
}
KINDS = 5      # pixels that differ


def repeated(g, layout, N, C, H, W, dtype):
    """A tensor whose pixels repeat KINDS different ones, and which of them each is."""
    which = torch.arange(N * H * W) % KINDS
    v = T.randn(g, KINDS, C)[which].view(N, H * W, C).permute(0, 2, 1).reshape(N, C, H, W)
    return T.put(layout, v, dtype)[0], which.cuda()


def all_equal(t, which, what):
    rows = t.float().permute(0, 2, 3, 1).reshape(-1, t.shape[1])
    first = rows[:KINDS][which]
    assert torch.equal(rows, first), (what, float((rows - first).abs().max()), int((rows != first).any(1).sum()))


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_pixel_s_bits_do_not_depend_on_its_place(name, dtype):
    (N, C, H, W, K), layout = SHAPES[name]
    g = T.rng(23)
    x, which = repeated(g, layout, N, C, H, W, dtype)
    w, b = (T.randn(g, 2 * K, C) / C ** 0.5).to(A.DT[dtype]).cuda(), B.vec(g, 2 * K)
    h, zg, zu = (A.tensor(layout, N, K, H, W, "f32")[0] for _ in range(3))
    dc.gate_fwd(V(x), x, w, b, dc.DC_ACT_GELU, None, V(zg), zg, zu, V(h), h)
    for t, what in ((zg, "zg"), (zu, "zu"), (h, "h")):
        all_equal(t, which, what)
    dy, _ = repeated(g, layout, N, C, H, W, dtype)
    w2 = (T.randn(g, C, K) / K ** 0.5).to(A.DT[dtype]).cuda()
    dz, again = (A.tensor(layout, N, c, H, W, "f32")[0] for c in (2 * K, K))
    dc.gate_bwd_data(V(dy), dy, w2, dc.DC_ACT_GELU, None, V(zg), zg, zu, V(again), again, V(dz), dz)
    all_equal(dz, which, "dz")
    all_equal(again, which, "h again")
