"""Layer norm, products over channels and 8-bit checkpoints against plain 64-bit
forms, at the layouts, sizes and values where they can go wrong.

Tolerances are bounds, not fits.  A sum of n fp32 terms in any order is within
n 2^-24 of the sum of their magnitudes; a result in bf16 within 2^-8 of itself
besides; what an activation adds is noted there.
"""
import numpy as np
import pytest
import torch

import act_ref as R
import paper_1903_06681_amd as dc

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def rng(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g)


def put(layout, values, dtype):
    """values [N][C][H][W] in a layout; the view and the memory around it (NaN)."""
    t, mem = R.tensor(layout, *values.shape, dtype)
    t.copy_(values.to("cuda"))
    return t, mem


def vec(g, n, mean=0.0):
    return (mean + 0.3 * randn(g, n)).cuda()


def ws(n):
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")


def ckpt(N, C, H, W):
    return ws(dc.ckpt_bytes(dc.View.q8(N, C, H, W)))


V = dc.View.of
# N, C, H, W: one value, one channel, ragged blocks, partial waves, many channels, long rows
TILES = [(1, 1, 1, 1), (2, 3, 1, 7), (1, 32, 5, 13), (3, 40, 9, 11), (2, 64, 16, 16), (1, 129, 3, 70),
         (2, 520, 4, 5), (1, 1030, 2, 3), (1, 2100, 1, 5), (1, 33, 40, 130)]
ROWS = [(1, 64, 1, 1), (5, 8, 1, 1), (70, 24, 1, 1), (33, 520, 1, 1), (3, 1032, 2, 1), (1, 4104, 3, 1), (2, 10, 3, 1)]
LAYOUTS = [(s, l) for s in TILES for l in ("dense", "padded", "gaps")] + [(s, l) for s in ROWS for l in ("rows", "slice", "dense")]


# ------------------------------------------------------------------ checkpoints

@pytest.mark.parametrize("shape,layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ckpt_save_and_load_bit_for_bit(shape, layout, dtype):
    N, C, H, W = shape
    g = rng(1)
    v = randn(g, *shape) * torch.exp2(torch.randint(-30, 30, (N, 1, H, W), generator=g).float())
    v.view(-1)[::7] = torch.round(v.view(-1)[::7])        # zeros and ties among them
    x, _ = put(layout, v, dtype)
    q = ckpt(*shape)
    dc.ckpt_save(V(x), x, q)
    want = R.q8_values(R.f64(x))
    np.testing.assert_array_equal(R.q8_decode(q, N, C, H * W), want)
    for out in ("f32", "bf16"):        # every value is exact in both
        y, mem = R.tensor(layout, *shape, out)
        dc.ckpt_load(dc.View.q8(*shape), q, dc.DC_ACT_NONE, V(y), y)
        np.testing.assert_array_equal(R.f64(y), want)
        assert R.untouched(y, mem)


def test_ckpt_takes_extremes_and_marks_what_is_not_finite():
    x = torch.zeros(1, 160, 1, 8)
    x[0, :32, 0, 0] = 0.0                                   # nothing
    x[0, 3, 0, 1] = 2.0 ** -149                             # below the least step: rounds to 0
    x[0, 4, 0, 2] = 2.0 ** -126 * 1.5                       # a tie: 1.5 steps, to even: 2
    x[0, 5, 0, 3] = 3.4028234e38                            # the largest
    x[0, 6, 0, 4] = -float("inf")
    x[0, 7, 0, 5] = float("nan")
    x[0, 40, 0, 4] = 1.0                                    # the next block of the same pixel stays
    x[0, 64:96, 0, 6] = torch.linspace(-1, 1, 32)
    x[0, 159, 0, 7] = -1.9999999
    t = x.cuda()
    q = ckpt(1, 160, 1, 8)
    dc.ckpt_save(V(t), t, q)
    got, want = R.q8_decode(q, 1, 160, 8), R.q8_values(R.f64(t))
    np.testing.assert_array_equal(got, want)
    assert np.isnan(got[0, :32, 4]).all() and np.isnan(got[0, :32, 5]).all() and got[0, 40, 4] == 1.0
    assert got[0, 5, 3] == 127 * 2.0 ** 121 and got[0, 159, 7] == -127 / 64
    y = torch.empty_like(t)
    dc.ckpt_load(dc.View.q8(1, 160, 1, 8), q, dc.DC_ACT_RELU, V(y), y)
    np.testing.assert_array_equal(R.f64(y), R.act(want, "relu"))


@pytest.mark.parametrize("kind", ["relu", "gelu", "silu"])
def test_ckpt_load_applies_the_activation(kind):
    """gelu's and silu's error: 7.1.26's 1.5e-7 of |z| and a few roundings of fp32."""
    z = torch.linspace(-12, 12, 32 * 25).view(1, 32, 5, 5).cuda()
    q = ckpt(1, 32, 5, 5)
    dc.ckpt_save(V(z), z, q)
    kept = R.q8_values(R.f64(z))
    y = torch.empty_like(z)
    dc.ckpt_load(dc.View.q8(1, 32, 5, 5), q, dc.ACT[kind], V(y), y)
    R.close(R.f64(y), R.act(kept, kind), 4e-7 * np.abs(kept) + 1e-12, kind)


# ------------------------------------------------------------------ layer norm

def norm_tol(x, mu, r, gamma, beta):
    """u: the mean and the centred values are within (C + 8) 2^-24 of the pixel's largest value,
    times r gamma; the variance's own error is relative and smaller still."""
    C = x.shape[1]
    top = np.abs(x).max(1, keepdims=True)
    xh = np.abs(x - mu) * r
    return R.EPS32 * np.abs(gamma)[:, None] * ((C + 8) * top * r * (1 + xh * xh.mean(1, keepdims=True)) + (C + 16) * xh) \
        + 2 * R.EPS32 * np.abs(beta)[:, None]


@pytest.mark.parametrize("shape,layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", ["f32-f32", "f32-bf16", "bf16-bf16", "bf16-f32"])
def test_norm_fwd(shape, layout, types):
    tx, tu = types.split("-")
    N, C, H, W = shape
    g = rng(2)
    x, _ = put(layout, 0.7 * randn(g, *shape) + randn(g, 1, C, 1, 1), tx)
    u, mem = R.tensor(layout, *shape, tu)
    gamma, beta = vec(g, C, 1.0), vec(g, C)
    stat, q = torch.empty(2, N, H, W, device="cuda"), ckpt(*shape)
    dc.norm_fwd(V(x), x, gamma, beta, EPS, V(u), u, stat, q)
    xs, ga, be = R.f64(x), gamma.cpu().double().numpy(), beta.cpu().double().numpy()
    want, mu, r = R.norm(xs, ga, be, EPS)
    tol = norm_tol(xs, mu, r, ga, be)
    R.close(R.f64(u), want, tol + (R.BF * np.abs(want) if tu == "bf16" else 0), "u")
    assert R.untouched(u, mem)
    top = np.abs(xs).max(1)
    st = stat.cpu().double().numpy().reshape(2, N, -1)
    R.close(st[0], mu[:, 0], (C + 2) * R.EPS32 * top, "mu")
    R.close(st[1], r[:, 0], R.EPS32 * r[:, 0] * (8 + C + (C + 8) * top * r[:, 0] * 2), "r")
    np.testing.assert_array_equal(R.q8_decode(q, N, C, H * W), R.q8_values(xs))


def test_norm_without_parameters_statistics_or_checkpoint_and_in_place():
    g = rng(3)
    x = (3 + randn(g, 2, 48, 6, 10)).cuda()
    xs = R.f64(x)
    want, mu, r = R.norm(xs, np.ones(48), np.zeros(48), EPS)
    u = torch.empty_like(x)
    dc.norm_fwd(V(x), x, None, None, EPS, V(u), u)
    R.close(R.f64(u), want, norm_tol(xs, mu, r, np.ones(48), np.zeros(48)), "u")
    dc.norm_fwd(V(x), x, None, None, EPS, V(x), x)
    assert torch.equal(x, u)


def test_norm_of_constant_and_offset_pixels():
    """No variance: u = beta exactly where the mean is exact; a mean of 2^12 spreads costs what the
    input's own 24 bits allow, not the squares' difference."""
    x = torch.full((1, 64, 1, 4), 0.5)
    x[0, :, 0, 1] = 0.0
    g = rng(4)
    x[0, :, 0, 2] = 4096 + randn(g, 64)
    t, beta = x.cuda(), vec(g, 64)
    u = torch.empty_like(t)
    dc.norm_fwd(V(t), t, None, beta, EPS, V(u), u)
    for p in (0, 1, 3):
        assert torch.equal(u[0, :, 0, p], beta) or p == 3
    xs = R.f64(t)
    want, mu, r = R.norm(xs, np.ones(64), beta.cpu().double().numpy(), EPS)
    R.close(R.f64(u), want, norm_tol(xs, mu, r, np.ones(64), beta.cpu().double().numpy()), "u")


@pytest.mark.parametrize("shape,layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", ["f32-f32-f32", "q8-bf16-bf16", "bf16-f32-bf16", "q8-f32-f32", "f32-bf16-f32"])
def test_norm_bwd(shape, layout, types):
    """Against the formula on the values that are kept; statistics are the forward's, handed over."""
    tx, tdu, to = types.split("-")
    N, C, H, W = shape
    g = rng(5)
    x, _ = put(layout, 0.7 * randn(g, *shape) + randn(g, 1, C, 1, 1), "bf16" if tx == "bf16" else "f32")
    du, _ = put(layout, randn(g, *shape), tdu)
    res, _ = put(layout, randn(g, *shape), to)
    dx, mem = R.tensor(layout, *shape, to)
    u, umem = R.tensor(layout, *shape, tdu)
    gamma, beta = vec(g, C, 1.0), vec(g, C)
    stat, q = torch.empty(2, N, H, W, device="cuda"), ckpt(*shape)
    dc.norm_fwd(V(x), x, gamma, beta, EPS, V(u), u, stat, q)
    vx, px = (dc.View.q8(*shape), q) if tx == "q8" else (V(x), x)
    xs = R.q8_decode(q, N, C, H * W) if tx == "q8" else R.f64(x)
    u.fill_(float("nan"))
    dg, db = vec(g, C), vec(g, C)
    dg0, db0 = dg.cpu().double().numpy(), db.cpu().double().numpy()
    need = dc.norm_bwd_workspace_bytes(V(du))
    dc.norm_bwd(V(du), du, vx, px, stat, gamma, beta, V(res), res, V(u), u, V(dx), dx, dg, db, 1, ws(need))
    ga, be = gamma.cpu().double().numpy(), beta.cpu().double().numpy()
    st = stat.cpu().double().numpy().reshape(2, N, 1, -1)
    dus, rs = R.f64(du), R.f64(res)
    want, wg, wb, xh = R.norm_bwd(dus, xs, st[0], st[1], ga)
    # xh: two roundings of the centred value's operands; sums of C products
    exh = 3 * R.EPS32 * st[1] * (np.abs(xs) + np.abs(st[0]))
    gd = np.abs(ga[:, None] * dus)
    m1, m2 = gd.mean(1, keepdims=True), (gd * np.abs(xh)).mean(1, keepdims=True)
    em2 = (C + 8) * R.EPS32 * m2 + (gd * exh).mean(1, keepdims=True)
    tol = st[1] * (8 * R.EPS32 * gd + (C + 8) * R.EPS32 * m1 + np.abs(xh) * em2 + (exh + 4 * R.EPS32 * np.abs(xh)) * m2)
    want = want + rs
    tol = tol + 2 * R.EPS32 * np.abs(want) + (R.BF * np.abs(want) if to == "bf16" else 0)
    R.close(R.f64(dx), want, tol, "dx")
    wu = ga[:, None] * xh + be[:, None]
    R.close(R.f64(u), wu, np.abs(ga)[:, None] * exh + 4 * R.EPS32 * (np.abs(wu) + np.abs(be)[:, None]) +
            (R.BF * np.abs(wu) if tdu == "bf16" else 0), "u")
    M = N * H * W
    R.close(dg.cpu().double().numpy(), dg0 + wg, (M + 4) * R.EPS32 * (np.abs(dus * xh).sum((0, 2)) + np.abs(dg0)) +
            (np.abs(dus) * exh).sum((0, 2)), "dgamma")
    R.close(db.cpu().double().numpy(), db0 + wb, (M + 4) * R.EPS32 * (np.abs(dus).sum((0, 2)) + np.abs(db0)), "dbeta")
    assert R.untouched(dx, mem) and R.untouched(u, umem)
    # overwriting, without a skip path, u or one of the parameters; the rest to the bit
    dx2, dg2 = torch.empty_like(dx), torch.empty_like(dg)
    dc.norm_bwd(V(du), du, vx, px, stat, gamma, None, None, None, None, None, V(dx2), dx2, dg2, None, 0, ws(need))
    R.close(R.f64(dx2), want - rs, tol + 2 * R.EPS32 * np.abs(rs) + (R.BF * np.abs(want - rs) if to == "bf16" else 0), "dx")
    R.close(dg2.cpu().double().numpy(), wg, (M + 4) * R.EPS32 * np.abs(dus * xh).sum((0, 2)) +
            (np.abs(dus) * exh).sum((0, 2)), "dgamma")


# between 512 and 2048 groups of 16 pixels (four of a row's): two to four a workgroup, one turn
TURNS = [((1, 40, 107, 93), "dense"), ((1, 70, 120, 161), "padded"), ((3, 56, 98, 97), "gaps"), ((9000, 100, 1, 1), "rows"),
         ((2500, 520, 1, 1), "slice")]


@pytest.mark.parametrize("shape,layout", TURNS, ids=str)
@pytest.mark.parametrize("types", ["f32-f32-f32", "q8-bf16-bf16"])
def test_norm_bwd_pixel_groups_of_a_workgroup(shape, layout, types):
    test_norm_bwd(shape, layout, types)


def test_norm_bwd_many_pixels_is_the_same_twice():
    """More pixel groups than workgroups: every workgroup takes several turns; fixed order."""
    g = rng(6)
    for C in (8, 64, 200):
        x, du = randn(g, 3, C, 150, 131).cuda(), randn(g, 3, C, 150, 131).cuda()
        u, dx, stat = torch.empty_like(x), torch.empty_like(x), torch.empty(2, 3, 150, 131, device="cuda")
        dc.norm_fwd(V(x), x, None, None, EPS, V(u), u, stat)
        out = []
        for _ in range(2):
            dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
            dc.norm_bwd(V(du), du, V(x), x, stat, None, None, None, None, None, None, V(dx), dx, dg, db, 0,
                        ws(dc.norm_bwd_workspace_bytes(V(du))))
            out.append((dx.clone(), dg, db))
        assert all(torch.equal(a, b) for a, b in zip(*out))
        xs, dus = R.f64(x), R.f64(du)
        st = stat.cpu().double().numpy().reshape(2, 3, 1, -1)
        want, wg, wb, xh = R.norm_bwd(dus, xs, st[0], st[1], np.ones(C))
        M = 3 * 150 * 131
        # random signs: errors add like a walk; 2^-24 (64 + M / 512 turns) per term is above any order used
        n = 128 + M / 512
        R.close(dg.cpu().double().numpy(), wg, n * R.EPS32 * np.abs(dus * xh).sum((0, 2)), "dgamma")
        R.close(db.cpu().double().numpy(), wb, n * R.EPS32 * np.abs(dus).sum((0, 2)), "dbeta")


def test_norm_keeps_what_is_not_finite_to_its_pixel():
    g = rng(7)
    x = randn(g, 1, 70, 4, 33)
    x[0, 5, 1, 2], x[0, 66, 3, 32] = float("inf"), float("nan")
    t = x.cuda()
    u, stat = torch.empty_like(t), torch.empty(2, 1, 4, 33, device="cuda")
    dc.norm_fwd(V(t), t, None, None, EPS, V(u), u, stat)
    bad = torch.zeros(4, 33, dtype=torch.bool)
    bad[1, 2] = bad[3, 32] = True
    assert torch.equal(torch.isfinite(u[0]).all(0).cpu(), ~bad)
    assert torch.equal((~torch.isfinite(u[0])).any(0).cpu(), bad)
    du, dx, dg = randn(g, 1, 70, 4, 33).cuda(), torch.empty_like(t), torch.empty(70, device="cuda")
    dc.norm_bwd(V(du), du, V(t), t, stat, None, None, None, None, None, None, V(dx), dx, dg, None, 0,
                ws(dc.norm_bwd_workspace_bytes(V(du))))
    assert torch.equal(torch.isfinite(dx[0]).all(0).cpu(), ~bad)


# ------------------------------------------------------------------ products

# N, C, H, W, K: single values, ragged blocks and slices, partial chunks, whole blocks
PRODUCTS = [(1, 1, 1, 1, 1), (2, 3, 1, 7, 5), (1, 32, 5, 13, 33), (3, 40, 9, 11, 72), (2, 64, 16, 16, 64), (1, 130, 3, 70, 129),
            (1, 257, 12, 20, 200), (5, 72, 7, 7, 260), (1, 16, 130, 140, 24), (2, 100, 40, 150, 150)]
PROWS = [(1, 64, 1, 1, 10), (3, 2050, 1, 1, 1000), (5, 8, 1, 1, 9), (70, 24, 1, 1, 40), (300, 136, 1, 1, 264), (3, 65, 20, 1, 31)]
PLAYOUTS = [(s, l) for s in PRODUCTS for l in ("dense", "padded", "gaps")] + [(s, l) for s in PROWS for l in ("rows", "slice", "dense")]


def linear_case(g, shape, layout, dtype, out=None):
    N, C, H, W, K = shape
    x, _ = put(layout, randn(g, N, C, H, W), dtype)
    w = (randn(g, K, C) / C ** 0.5).to(R.DT[dtype]).cuda()
    b = vec(g, K)
    return x, w, b


def product(w, x):
    w = w.cpu().double().numpy()
    return np.einsum("kc,ncp->nkp", w, x), np.einsum("kc,ncp->nkp", np.abs(w), np.abs(x))


@pytest.mark.parametrize("shape,layout", PLAYOUTS, ids=str)
@pytest.mark.parametrize("dtype,out,act,res", [("f32", "f32", "gelu", None), ("bf16", "bf16", "gelu", "bf16"), ("bf16", "f32", "none", "f32"),
                                               ("bf16", "bf16", "silu", None), ("f32", "bf16", "relu", "f32")])
def test_linear_fwd(shape, layout, dtype, out, act, res):
    N, C, H, W, K = shape
    g = rng(11)
    x, w, b = linear_case(g, shape, layout, dtype)
    y, mem = R.tensor(layout, N, K, H, W, out)
    r, vr = None, None
    if res:
        r, _ = put(layout, randn(g, N, K, H, W), res)
        vr = V(r)
    dc.linear_fwd(V(x), x, w, b, dc.ACT[act], vr, r, None, None, V(y), y)
    z, top = product(w, R.f64(x))
    z, top = z + b.cpu().double().numpy()[:, None], top + np.abs(b.cpu().double().numpy())[:, None]
    want = R.act(z, act) + (R.f64(r) if res else 0)
    # slopes are at most 1.13; the activation itself adds 4e-7 |z|, the residual's sum a rounding
    tol = 1.13 * (C + 2) * R.EPS32 * top + 4e-7 * np.abs(z) + 2 * R.EPS32 * np.abs(want) + \
        (R.BF * np.abs(want) if out == "bf16" else 0)
    R.close(R.f64(y), want, tol, "y")
    assert R.untouched(y, mem)


# long sums with 54 to 64 blocks of 64 x 64 results to share them
FEW = [((2, 300, 23, 29, 130), "dense"), ((1, 1030, 33, 31, 200), "gaps"), ((1100, 260, 1, 1, 130), "rows"), ((1100, 263, 1, 1, 130), "slice")]


@pytest.mark.parametrize("shape,layout", FEW, ids=str)
@pytest.mark.parametrize("dtype,out,act,res", [("f32", "f32", "gelu", "f32"), ("bf16", "bf16", "silu", "bf16")])
def test_linear_fwd_long_sums_few_blocks(shape, layout, dtype, out, act, res):
    test_linear_fwd(shape, layout, dtype, out, act, res)


@pytest.mark.parametrize("shape,layout", PLAYOUTS, ids=str)
@pytest.mark.parametrize("dtype,keep,act", [("f32", "f32", "gelu"), ("bf16", "q8", "gelu"), ("bf16", "bf16", "silu"), ("f32", "q8", "relu")])
def test_linear_kept_activation_and_its_gradient(shape, layout, dtype, keep, act):
    """z as the forward pass keeps it, then (W2^T dy) act'(z) and act(z) from what was kept."""
    N, C, H, W, K = shape
    P = H * W
    g = rng(12)
    x, w, b = linear_case(g, shape, layout, dtype)
    h, hmem = R.tensor(layout, N, K, H, W, dtype)
    if keep == "q8":
        kz, vz = ckpt(N, K, H, W), dc.View.q8(N, K, H, W)
    else:
        kz, zmem = R.tensor(layout, N, K, H, W, keep)
        vz = V(kz)
    dc.linear_fwd(V(x), x, w, b, dc.ACT[act], None, None, vz, kz, V(h), h)
    z, top = product(w, R.f64(x))
    bd = b.cpu().double().numpy()[:, None]
    z, top = z + bd, top + np.abs(bd)
    ez = (C + 2) * R.EPS32 * top
    if keep == "q8":
        zs = R.q8_decode(kz, N, K, P)
        full = np.zeros((N, -(-K // 32) * 32, P))
        full[:, :K] = np.abs(z)
        power = 2.0 ** np.floor(np.log2(np.maximum(full.reshape(N, -1, 32, P).max(2), 2.0 ** -120)))
        # half a step of 2^-6 of the power (a whole one at the very top); the power itself may round up
        R.close(zs, z, 2.0 ** -6 * np.repeat(power, 32, 1)[:, :K] * (1 + 1e-5) + ez, "z8")
    else:
        zs = R.f64(kz)
        R.close(zs, z, ez + (R.BF * np.abs(z) if keep == "bf16" else 0), "z")
        assert R.untouched(kz, zmem)
    # the input gradient of a product [C][K] after it
    dy, _ = put(layout, randn(g, N, C, H, W), dtype)
    w2 = (randn(g, C, K) / K ** 0.5).to(R.DT[dtype]).cuda()
    dz, mem = R.tensor(layout, N, K, H, W, dtype)
    h.fill_(float("nan"))
    dc.linear_bwd_data(V(dy), dy, w2, dc.ACT[act], vz, kz, V(h), h, V(dz), dz)
    p, ptop = product(w2.t(), R.f64(dy))
    sl = R.slope(zs, act)
    want, wh = p * sl, R.act(zs, act)
    rnd = R.BF if dtype == "bf16" else 0
    # the slope's own error: 1.5e-7 and a few roundings of values up to 1.13
    R.close(R.f64(dz), want, 1.13 * (C + 2) * R.EPS32 * ptop + 1e-6 * np.abs(p) + (rnd + 2 * R.EPS32) * np.abs(want), "dz")
    R.close(R.f64(h), wh, 4e-7 * np.abs(zs) + (rnd + 2 * R.EPS32) * np.abs(wh), "h")
    assert R.untouched(dz, mem) and R.untouched(h, hmem)
    # without an activation: the plain input gradient
    dc.linear_bwd_data(V(dy), dy, w2, dc.DC_ACT_NONE, None, None, None, None, V(dz), dz)
    R.close(R.f64(dz), p, (C + 2) * R.EPS32 * ptop + rnd * np.abs(p), "dx")


@pytest.mark.parametrize("shape,layout", PLAYOUTS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_bwd_filter(shape, layout, dtype):
    N, C, H, W, K = shape
    g = rng(13)
    x, _ = put(layout, randn(g, N, C, H, W), dtype)
    dy, _ = put(layout, randn(g, N, K, H, W), dtype)
    dw, db = vec(g, K * C).view(K, C).clone(), vec(g, K)
    dw0, db0 = dw.cpu().double().numpy(), db.cpu().double().numpy()
    need = dc.linear_bwd_filter_workspace_bytes(V(x), V(dy))
    dc.linear_bwd_filter(V(x), x, V(dy), dy, dw, db, 1, ws(need))
    xs, ys = R.f64(x), R.f64(dy)
    want, top = np.einsum("nkp,ncp->kc", ys, xs), np.einsum("nkp,ncp->kc", np.abs(ys), np.abs(xs))
    M = N * H * W
    R.close(dw.cpu().double().numpy(), dw0 + want, (M + 4) * R.EPS32 * (top + np.abs(dw0)), "dw")
    R.close(db.cpu().double().numpy(), db0 + ys.sum((0, 2)), (M + 4) * R.EPS32 * (np.abs(ys).sum((0, 2)) + np.abs(db0)), "db")
    dw2 = torch.full((K, C), float("nan"), device="cuda")
    dc.linear_bwd_filter(V(x), x, V(dy), dy, dw2, None, 0, ws(need))
    R.close(dw2.cpu().double().numpy(), want, (M + 4) * R.EPS32 * top, "dw")
    again = torch.empty_like(dw2)
    dc.linear_bwd_filter(V(x), x, V(dy), dy, again, db, 0, ws(need))
    assert torch.equal(again, dw2)
    R.close(db.cpu().double().numpy(), ys.sum((0, 2)), (M + 4) * R.EPS32 * np.abs(ys).sum((0, 2)), "db")


@pytest.mark.parametrize("shape,layout", [((2100, 1090, 1, 1, 1010), "rows"), ((1, 1090, 42, 51, 1010), "padded")], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_bwd_filter_two_shares(shape, layout, dtype):
    """288 blocks of 64 x 64 results, 33 slices and more."""
    test_linear_bwd_filter(shape, layout, dtype)


# N, C, H, W, K: the largest blocks with whole slices, with a ragged end of everything (rows
# off the alignment), results stored past the caches, a single slice
LARGE = [(2, 136, 128, 128, 512), (1, 257, 181, 183, 515), (1, 64, 300, 300, 264), (1, 24, 512, 522, 40)]


@pytest.mark.parametrize("shape", LARGE, ids=str)
@pytest.mark.parametrize("dtype,keep", [("f32", "f32"), ("bf16", "q8"), ("bf16", "f32")])
def test_linear_large_blocks(shape, dtype, keep):
    """As above, the references summed in 64 bits on the GPU."""
    N, C, H, W, K = shape
    g = torch.Generator(device="cuda")
    g.manual_seed(18)

    def dev(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def rows(t):
        return t.permute(1, 0, 2, 3).reshape(t.shape[1], -1).double()

    def near(got, want, tol, what):
        bad = (rows(got) - want).abs() - tol
        assert not bool((bad > 0).any()), (what, float(bad.max()))

    dt, rnd = R.DT[dtype], R.BF if dtype == "bf16" else 0
    x, w, b, res = dev(N, C, H, W).to(dt), (dev(K, C) / C ** 0.5).to(dt), 0.3 * dev(K), dev(N, K, H, W).to(dt)
    y = torch.full((N, K, H, W), float("nan"), dtype=dt, device="cuda")
    h, dz = torch.empty_like(y), torch.empty_like(y)
    kz = ckpt(N, K, H, W) if keep == "q8" else torch.empty(N, K, H, W, device="cuda")
    vz = dc.View.q8(N, K, H, W) if keep == "q8" else V(kz)
    dc.linear_fwd(V(x), x, w, b, dc.DC_ACT_SILU, V(res), res, vz, kz, V(y), y)
    z, top = w.double() @ rows(x) + b.double()[:, None], w.double().abs() @ rows(x).abs() + b.double().abs()[:, None]
    want = z * torch.sigmoid(z) + rows(res)
    near(y, want, 1.13 * (C + 2) * R.EPS32 * top + 4e-7 * z.abs() + (rnd + 2 * R.EPS32) * want.abs(), "y")
    if keep == "q8":
        zf = torch.empty(N, K, H, W, device="cuda")
        dc.ckpt_load(vz, kz, dc.DC_ACT_NONE, V(zf), zf)
        full = torch.zeros(-(-K // 32) * 32, N * H * W, dtype=torch.float64, device="cuda")
        full[:K] = z.abs()
        power = torch.exp2(torch.floor(torch.log2(full.view(-1, 32, N * H * W).amax(1))))
        near(zf, z, 2.0 ** -6 * power.repeat_interleave(32, 0)[:K] * (1 + 1e-5) + (C + 2) * R.EPS32 * top, "z8")
        zs = rows(zf)
    else:
        near(kz, z, (C + 2) * R.EPS32 * top, "z")
        zs = rows(kz)
    dy, w2 = dev(N, C, H, W).to(dt), (dev(C, K) / K ** 0.5).to(dt)
    dc.linear_bwd_data(V(dy), dy, w2, dc.DC_ACT_SILU, vz, kz, V(h), h, V(dz), dz)
    p, ptop, sg = w2.double().t() @ rows(dy), w2.double().abs().t() @ rows(dy).abs(), torch.sigmoid(zs)
    want = p * sg * (1 + zs * (1 - sg))
    near(dz, want, 1.13 * (C + 2) * R.EPS32 * ptop + 1e-6 * p.abs() + (rnd + 2 * R.EPS32) * want.abs(), "dz")
    near(h, zs * sg, 4e-7 * zs.abs() + (rnd + 2 * R.EPS32) * (zs * sg).abs(), "h")
    dw, db = torch.empty(K, C, device="cuda"), torch.empty(K, device="cuda")
    dc.linear_bwd_filter(V(x), x, V(res), res, dw, db, 0, ws(dc.linear_bwd_filter_workspace_bytes(V(x), V(res))))
    want, top = rows(res) @ rows(x).t(), rows(res).abs() @ rows(x).abs().t()
    # slices, shares and lanes cut the sum of N H W terms in pieces of at most 4096
    assert bool(((dw.double() - want).abs() <= 4096 * R.EPS32 * top).all())
    assert bool(((db.double() - rows(res).sum(1)).abs() <= 4096 * R.EPS32 * rows(res).abs().sum(1)).all())


def test_linear_mixed_layouts():
    """Rows of channels in, a tile out, and the other way: one view decides nothing for the others."""
    g = rng(14)
    for lx, ly, shape in (("rows", "dense", (7, 40, 6, 1)), ("dense", "rows", (7, 40, 6, 1)), ("slice", "gaps", (3, 136, 5, 1)),
                          ("gaps", "rows", (2, 72, 9, 1))):
        N, C, H, W = shape
        for dtype in ("f32", "bf16"):
            x, _ = put(lx, randn(g, *shape), dtype)
            w = (randn(g, 50, C) / C ** 0.5).to(R.DT[dtype]).cuda()
            y, mem = R.tensor(ly, N, 50, H, W, "f32")
            dc.linear_fwd(V(x), x, w, None, dc.DC_ACT_NONE, None, None, None, None, V(y), y)
            z, top = product(w, R.f64(x))
            R.close(R.f64(y), z, (C + 2) * R.EPS32 * top, "y")
            assert R.untouched(y, mem)
            dw = torch.empty(50, C, device="cuda")
            dy, _ = put(ly, randn(g, N, 50, H, W), dtype)
            dc.linear_bwd_filter(V(x), x, V(dy), dy, dw, None, 0, ws(dc.linear_bwd_filter_workspace_bytes(V(x), V(dy))))
            xs, ys = R.f64(x), R.f64(dy)
            R.close(dw.cpu().double().numpy(), np.einsum("nkp,ncp->kc", ys, xs),
                    (N * H + 4) * R.EPS32 * np.einsum("nkp,ncp->kc", np.abs(ys), np.abs(xs)), "dw")


def test_linear_broadcast_input_and_residual():
    """Strides of 0 in what is read: one row of channels for every pixel, one residual for every sample."""
    g = rng(15)
    x = randn(g, 1, 24, 1, 1).cuda().expand(3, 24, 4, 1)
    w, res = randn(g, 20, 24).cuda(), randn(g, 1, 20, 4, 1).cuda().expand(3, 20, 4, 1)
    y = torch.empty(3, 20, 4, 1, device="cuda")
    dc.linear_fwd(V(x), x, w, None, dc.DC_ACT_NONE, V(res), res, None, None, V(y), y)
    z, top = product(w, R.f64(x))
    want = z + R.f64(res)
    R.close(R.f64(y), want, 26 * R.EPS32 * top + R.EPS32 * np.abs(want), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_keeps_what_is_not_finite_to_its_pixel(dtype):
    g = rng(16)
    x = randn(g, 2, 70, 6, 21)
    x[0, 5, 1, 2], x[1, 66, 3, 20] = float("inf"), float("nan")
    t = x.to(R.DT[dtype]).cuda()
    w = randn(g, 90, 70).to(R.DT[dtype]).cuda()
    y = torch.empty(2, 90, 6, 21, device="cuda")
    dc.linear_fwd(V(t), t, w, None, dc.DC_ACT_NONE, None, None, None, None, V(y), y)
    want, _ = product(w, R.f64(t))
    got = R.f64(y)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    dy = randn(g, 2, 90, 6, 21).to(R.DT[dtype]).cuda()
    dw = torch.empty(90, 70, device="cuda")
    dc.linear_bwd_filter(V(t), t, V(dy), dy, dw, None, 0, ws(dc.linear_bwd_filter_workspace_bytes(V(t), V(dy))))
    want = np.einsum("nkp,ncp->kc", R.f64(dy), R.f64(t))
    got = dw.cpu().double().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])


def test_offsets_past_32_bits():
    """A view whose last sample starts more than 2^32 bytes and 2^31 elements in."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 20 GB of the card")
    g = rng(17)
    mem = torch.empty((1 << 31) + (1 << 20), dtype=torch.float32, device="cuda")
    shape, far = (2, 40, 6, 20), 1 << 31
    x = torch.as_strided(mem, shape, (far, 6 * 20, 20, 1))
    x.copy_(randn(g, *shape))
    w = randn(g, 24, 40).cuda()
    ymem = torch.empty((1 << 31) + (1 << 20), dtype=torch.float32, device="cuda")
    y = torch.as_strided(ymem, (2, 24, 6, 20), (far, 120, 20, 1))
    dc.linear_fwd(V(x), x, w, None, dc.DC_ACT_NONE, None, None, None, None, V(y), y)
    z, top = product(w, R.f64(x.contiguous()))
    R.close(R.f64(y.contiguous()), z, 42 * R.EPS32 * top, "y")
    dw = torch.empty(24, 40, device="cuda")
    dc.linear_bwd_filter(V(x), x, V(y), y, dw, None, 0, ws(dc.linear_bwd_filter_workspace_bytes(V(x), V(y))))
    xs, ys = R.f64(x.contiguous()), R.f64(y.contiguous())
    R.close(dw.cpu().double().numpy(), np.einsum("nkp,ncp->kc", ys, xs),
            244 * R.EPS32 * np.einsum("nkp,ncp->kc", np.abs(ys), np.abs(xs)), "dw")
    u = torch.as_strided(ymem, shape, (far, 120, 20, 1))
    stat, q = torch.empty(2, 2, 6, 20, device="cuda"), ckpt(*shape)
    dc.norm_fwd(V(x), x, None, None, EPS, V(u), u, stat, q)
    want, mu, r = R.norm(xs, np.ones(40), np.zeros(40), EPS)
    R.close(R.f64(u.contiguous()), want, norm_tol(xs, mu, r, np.ones(40), np.zeros(40)), "u")
    np.testing.assert_array_equal(R.q8_decode(q, 2, 40, 120), R.q8_values(xs))


# ------------------------------------------------------------------ streams and graphs

def _block(s):
    """A block's forward and backward on the current stream, outputs in place."""
    dc.norm_fwd(V(s["x"]), s["x"], s["gamma"], s["beta"], EPS, V(s["u"]), s["u"], s["stat"], s["qx"])
    dc.linear_fwd(V(s["u"]), s["u"], s["w1"], s["b1"], dc.DC_ACT_GELU, None, None, s["vq"], s["qz"], V(s["h"]), s["h"])
    dc.linear_fwd(V(s["h"]), s["h"], s["w2"], s["b2"], dc.DC_ACT_NONE, V(s["x"]), s["x"], None, None, V(s["y"]), s["y"])
    dc.linear_bwd_data(V(s["y"]), s["y"], s["w2"], dc.DC_ACT_GELU, s["vq"], s["qz"], V(s["h"]), s["h"], V(s["dz"]), s["dz"])
    dc.linear_bwd_filter(V(s["h"]), s["h"], V(s["y"]), s["y"], s["dw2"], s["db2"], 0, s["ws2"])
    dc.linear_bwd_data(V(s["dz"]), s["dz"], s["w1"], dc.DC_ACT_NONE, None, None, None, None, V(s["du"]), s["du"])
    dc.norm_bwd(V(s["du"]), s["du"], s["vqx"], s["qx"], s["stat"], s["gamma"], s["beta"], V(s["y"]), s["y"], V(s["u"]), s["u"],
                V(s["dx"]), s["dx"], s["dgamma"], s["dbeta"], 0, s["wsn"])
    dc.linear_bwd_filter(V(s["u"]), s["u"], V(s["dz"]), s["dz"], s["dw1"], s["db1"], 0, s["ws1"])


def _state(seed):
    g, N, C, H, W, F = rng(seed), 2, 48, 13, 30, 96
    bf = torch.bfloat16
    s = {"x": randn(g, N, C, H, W).to(bf).cuda(), "gamma": vec(g, C, 1), "beta": vec(g, C), "b1": vec(g, F), "b2": vec(g, C),
         "w1": (randn(g, F, C) / 7).to(bf).cuda(), "w2": (randn(g, C, F) / 10).to(bf).cuda()}
    for n in ("u", "y", "du", "dx"):
        s[n] = torch.empty(N, C, H, W, dtype=bf, device="cuda")
    for n in ("h", "dz"):
        s[n] = torch.empty(N, F, H, W, dtype=bf, device="cuda")
    s["stat"] = torch.empty(2, N, H, W, device="cuda")
    s["vq"], s["vqx"] = dc.View.q8(N, F, H, W), dc.View.q8(N, C, H, W)
    s["qz"], s["qx"] = ckpt(N, F, H, W), ckpt(N, C, H, W)
    s["dgamma"], s["dbeta"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    s["dw1"], s["db1"] = torch.empty(F, C, device="cuda"), torch.empty(F, device="cuda")
    s["dw2"], s["db2"] = torch.empty(C, F, device="cuda"), torch.empty(C, device="cuda")
    s["ws1"] = ws(dc.linear_bwd_filter_workspace_bytes(V(s["u"]), V(s["dz"])))
    s["ws2"] = ws(dc.linear_bwd_filter_workspace_bytes(V(s["h"]), V(s["y"])))
    s["wsn"] = ws(dc.norm_bwd_workspace_bytes(V(s["du"])))
    return s


OUT = ("y", "dz", "h", "dx", "u", "dgamma", "dbeta", "dw1", "db1", "dw2", "db2")


def test_block_on_another_stream_and_in_a_graph():
    """The same bits on a side stream and in every replay of a graph, eager work between the replays."""
    s = _state(21)
    _block(s)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in OUT}
    assert all(bool(torch.isfinite(want[n].float()).all()) for n in OUT)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _block(s)
    side.synchronize()
    assert all(torch.equal(s[n], want[n]) for n in OUT)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _block(s)
    x = s["x"].clone()
    for k in range(4):
        other = _state(30 + k)
        _block(other)
        s["x"].copy_(other["x"] if k % 2 else x)
        for n in OUT:
            s[n].fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: s[n].clone() for n in OUT}
        _block(s)
        torch.cuda.synchronize()
        assert all(torch.equal(s[n], got[n]) for n in OUT), k
        if k % 2 == 0:
            assert all(torch.equal(got[n], want[n]) for n in OUT), k
