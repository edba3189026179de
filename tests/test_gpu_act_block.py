"""The example that runs the operators between two decomposed convolutions: its gradients
against automatic differentiation of the same network on the whole image in 64 bits, and
its training."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import tile_block
    return tile_block


def whole(tiles, grid):
    """[grid grid N][C][h][w] -> [N][C][H][W]."""
    B, C, h, w = tiles.shape
    N = B // (grid * grid)
    return tiles.view(grid, grid, N, C, h, w).permute(2, 3, 0, 4, 1, 5).reshape(N, C, grid * h, grid * w)


def test_gradients_of_the_block_against_the_whole_image(block):
    """Each tensor is rounded to 8 significant bits a few times (bf16) and the activations kept
    for the backward pass to 7 (8-bit checkpoints): relative errors of 2^-8 and 2^-7 at most
    each, which average out over a gradient's sum.  A gradient's error over its own length has
    to stay below 2^-5; a term left out or taken twice would be of order one."""
    b = block.TileBlock(N=1, C=5, width=40, hidden=96, out=7, size=24, grid=2, seed=3)
    g = torch.Generator().manual_seed(4)
    for k in ("gamma", "beta", "b1", "b2"):
        b.params[k] += 0.3 * torch.randn(b.params[k].shape, generator=g).cuda()
    x, dy = torch.randn(1, 5, 24, 24, generator=g), torch.randn(4, 7, 12, 12, generator=g)
    y = b.forward(x.cuda())
    got = {k: v.cpu().double() for k, v in b.backward(dy.cuda()).items()}
    F = torch.nn.functional
    p = {k: (b.w[k] if k in b.w else v).detach().cpu().double().requires_grad_() for k, v in b.params.items()}
    a = F.conv2d(x.to(torch.bfloat16).double(), p["c1"], padding=1)
    u = F.layer_norm(a.permute(0, 2, 3, 1), (40,), p["gamma"], p["beta"], 1e-5)
    o = a + (F.gelu(u @ p["w1"].t() + p["b1"]) @ p["w2"].t() + p["b2"]).permute(0, 3, 1, 2)
    want = F.conv2d(o, p["c2"], padding=1)
    assert (whole(y.cpu().double(), 2) - want).norm() < 2 ** -5 * want.norm()
    want.backward(whole(dy.double(), 2))
    for k in p:
        err = float((got[k] - p[k].grad).norm() / p[k].grad.norm())
        print(f"{k}: {err:.4f}")
        assert err < 2 ** -5, k


def test_the_example_trains(block):
    losses = block.main(12)
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0]
    assert block.main(12) == losses                            # the same bits again
