"""Every kernel that the sizes pick, at sizes that pick it: the layer norm of whole tiles (64
pixels a wave) with one and two blocks a lane, many turns of the kernels that read a row again,
and the products' larger blocks over rows of channels and over tiles off the alignment.
References in 64 bits; bounds as in the tests of the same calls at small sizes."""
import pytest
import torch

import act_ref as R
import paper_1903_06681_amd as dc
import test_gpu_act as T

pytestmark = pytest.mark.gpu
V = dc.View.of
_gpu = T._gpu

# waves of 64 pixels and 32 channels: 2048 and more; 8 blocks and fewer a lane's one, 9 to 16 its two
NORM_TILES = [((1, 40, 300, 231), "dense"), ((1, 40, 300, 231), "gaps"), ((1, 300, 121, 123), "padded"), ((1, 512, 120, 101), "dense"),
              ((3, 24, 209, 211), "gaps")]
# rows and tiles of too many channels for the registers, several turns a workgroup
NORM_TURNS = [((1500, 4104, 1, 1), "rows"), ((1, 1056, 70, 73), "dense")]


def picked(shape):
    """Pixels of a wave, blocks a lane holds, for tiles."""
    N, C, H, W = shape
    blocks = -(-C // 32)
    return 64 if blocks <= 16 and -(-N * H * W // 64) * blocks >= 2048 else 16, -(-blocks // 8)


def test_the_sizes_pick_the_kernels_of_whole_tiles():
    assert {picked(s) for s, _ in NORM_TILES} == {(64, 1), (64, 2)}


@pytest.mark.parametrize("shape,layout", NORM_TILES + NORM_TURNS, ids=str)
@pytest.mark.parametrize("types", ["f32-f32", "f32-bf16", "bf16-bf16"])
def test_norm_fwd(shape, layout, types):
    T.test_norm_fwd(shape, layout, types)


@pytest.mark.parametrize("shape,layout", NORM_TILES + NORM_TURNS, ids=str)
@pytest.mark.parametrize("types", ["f32-f32-f32", "q8-bf16-bf16", "bf16-f32-bf16"])
def test_norm_bwd(shape, layout, types):
    T.test_norm_bwd(shape, layout, types)


# N, C, H, W, K, layout, block of the forward pass and the input gradient (bf16, fp32), of the weight gradient
PRODUCTS = {
    "middle_off_16_bytes": ((1, 100, 300, 301, 264), "dense"), "middle": ((1, 128, 300, 304, 264), "dense"),
    "middle_gaps": ((2, 72, 211, 150, 200), "gaps"), "short_padded": ((2, 32, 200, 250, 136), "padded"),
    "large_padded": ((2, 136, 130, 131, 512), "padded"), "large_gradient": ((2, 256, 256, 256, 512), "dense"),
    "rows_short": ((33000, 32, 1, 1, 264), "rows"), "rows_short_64": ((33000, 64, 1, 1, 264), "rows"),
    "rows_middle": ((33000, 100, 1, 1, 264), "rows"), "rows_middle_slice": ((35, 128, 1000, 1, 264), "slice"),
    "rows_large": ((70000, 264, 1, 1, 520), "rows"), "rows_large_ragged": ((70000, 263, 1, 1, 517), "slice"),
}


def block(rows, red, slots, bf16):
    def count(r, c):
        return -(-rows // r) * -(-slots // c)
    if red > 128 and count(256, 256) >= 256:
        return "large"
    return "small" if count(64, 128) < 512 else "short" if red <= (64 if bf16 else 32) else "middle"


def test_the_sizes_pick_the_blocks():
    for name, ((N, C, H, W, K), _) in PRODUCTS.items():
        kinds = [block(K, C, N * H * W, b) for b in (True, False)]
        assert any(k in name for k in kinds), (name, kinds)


@pytest.mark.parametrize("name", PRODUCTS)
@pytest.mark.parametrize("dtype,keep,act", [("f32", "f32", "gelu"), ("bf16", "q8", "silu"), ("bf16", "bf16", "gelu")])
def test_products(name, dtype, keep, act):
    """Forward with a residual and what the activation read, its gradient, the weights' and the bias's."""
    (N, C, H, W, K), layout = PRODUCTS[name]
    dt, rnd = R.DT[dtype], R.BF if dtype == "bf16" else 0
    g = torch.Generator(device="cuda")
    g.manual_seed(31)

    def dev(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def filled(channels, d=dtype):
        t, mem = R.tensor(layout, N, channels, H, W, d)
        t.copy_(dev(N, channels, H, W))
        return t, mem

    def rows(t):
        return t.permute(1, 0, 2, 3).reshape(t.shape[1], -1).double()

    def near(got, want, tol, what):
        bad = (rows(got) - want).abs() - tol
        assert not bool((bad > 0).any()) and not bool(torch.isnan(bad).any()), (what, float(bad.max()))

    def value(z):
        return z * torch.sigmoid(z) if act == "silu" else z * torch.special.ndtr(z)

    (x, _), (res, _), w, b = filled(C), filled(K), (dev(K, C) / C ** 0.5).to(dt), 0.3 * dev(K)
    y, ymem = R.tensor(layout, N, K, H, W, dtype)
    kz, zmem = (T.ckpt(N, K, H, W), None) if keep == "q8" else R.tensor(layout, N, K, H, W, keep)
    vz = dc.View.q8(N, K, H, W) if keep == "q8" else V(kz)
    dc.linear_fwd(V(x), x, w, b, dc.ACT[act], V(res), res, vz, kz, V(y), y)
    xs = rows(x)
    z, top = w.double() @ xs + b.double()[:, None], w.double().abs() @ xs.abs() + b.double().abs()[:, None]
    want = value(z) + rows(res)
    near(y, want, 1.13 * (C + 2) * R.EPS32 * top + 4e-7 * z.abs() + (rnd + 2 * R.EPS32) * want.abs(), "y")
    assert R.untouched(y, ymem)
    if keep == "q8":
        kept = torch.empty(N, K, H, W, device="cuda")
        dc.ckpt_load(vz, kz, dc.DC_ACT_NONE, V(kept), kept)
        blocks = torch.zeros(-(-K // 32) * 32, N * H * W, dtype=torch.float64, device="cuda")
        blocks[:K] = z.abs()
        power = torch.exp2(torch.floor(torch.log2(blocks.view(-1, 32, N * H * W).amax(1))))
        near(kept, z, 2.0 ** -6 * power.repeat_interleave(32, 0)[:K] * (1 + 1e-5) + (C + 2) * R.EPS32 * top, "z8")
        zs = rows(kept)
    else:
        near(kz, z, (C + 2) * R.EPS32 * top + (rnd if keep == "bf16" else 0) * z.abs(), "z")
        assert R.untouched(kz, zmem)
        zs = rows(kz)
    (dy, _), w2 = filled(C), (dev(C, K) / K ** 0.5).to(dt)
    (h, hmem), (dz, dmem) = R.tensor(layout, N, K, H, W, dtype), R.tensor(layout, N, K, H, W, dtype)
    dc.linear_bwd_data(V(dy), dy, w2, dc.ACT[act], vz, kz, V(h), h, V(dz), dz)
    ds = rows(dy)
    p, ptop = w2.double().t().contiguous() @ ds, w2.double().abs().t().contiguous() @ ds.abs()
    sg = torch.sigmoid(zs)
    slope = sg * (1 + zs * (1 - sg)) if act == "silu" else torch.special.ndtr(zs) + zs * torch.exp(-zs * zs / 2) * 0.3989422804014327
    want = p * slope
    near(dz, want, 1.13 * (C + 2) * R.EPS32 * ptop + 1e-6 * p.abs() + (rnd + 2 * R.EPS32) * want.abs(), "dz")
    near(h, value(zs), 4e-7 * zs.abs() + (rnd + 2 * R.EPS32) * value(zs).abs(), "h")
    assert R.untouched(h, hmem) and R.untouched(dz, dmem)
    # pieces of at most 4096 terms each, as the slices, shares and lanes cut the sum
    dw, db = torch.empty(K, C, device="cuda"), torch.empty(K, device="cuda")
    dc.linear_bwd_filter(V(x), x, V(res), res, dw, db, 0, T.ws(dc.linear_bwd_filter_workspace_bytes(V(x), V(res))))
    rs = rows(res)
    want, top = rs @ xs.t().contiguous(), rs.abs() @ xs.abs().t().contiguous()
    assert bool(((dw.double() - want).abs() <= 4096 * R.EPS32 * top).all())
    assert bool(((db.double() - rs.sum(1)).abs() <= 4096 * R.EPS32 * rs.abs().sum(1)).all())
