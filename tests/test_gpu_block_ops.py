"""A gated residual block's operators (the gated product, the join of a branch with its residual
stream, dropout) against plain 64-bit forms, at the layouts, sizes and values where they can go
wrong.  Bounds: block_ref.py; a result in bf16 is within 2^-8 of itself besides."""
import numpy as np
import pytest
import torch

import act_ref as A
import block_ref as R
import paper_1903_06681_amd as dc
import test_gpu_act as T

pytestmark = pytest.mark.gpu
V = dc.View.of
EPS = 1e-5
_gpu = T._gpu
put, rng, randn, ws, ckpt = T.put, T.rng, T.randn, T.ws, T.ckpt


def vec(g, *shape, mean=0.0):
    return (mean + 0.3 * randn(g, *shape)).cuda()


def f64(t):
    return t.double().reshape(t.shape[0], t.shape[1], -1)


def rnd(t):
    return R.BF if t.dtype == torch.bfloat16 else 0.0


def near(got, want, bound, what):
    """Within the bound, and the rounding of the tensor's own type."""
    w = want.reshape(f64(got).shape) if got.dim() == 4 else want
    g = f64(got) if got.dim() == 4 else got.double()
    bad = (g - w).abs() - (bound + rnd(got) * (w.abs() + bound))
    assert not bool(torch.isnan(bad).any()) and not bool((bad > 0).any()), (what, float(bad.max()), float((g - w).abs().max()))


def decode(q, N, C, H, W):
    return torch.from_numpy(A.q8_decode(q, N, C, H * W)).cuda()


# ------------------------------------------------------------------ dropout

PLACES = [{}, {"n0": 3, "h0": 2, "w0": 5, "H": 300, "W": 301, "offset": 2 ** 63 + 11}]


@pytest.mark.parametrize("shape,layout", T.LAYOUTS, ids=str)
@pytest.mark.parametrize("types", ["f32-f32", "bf16-bf16", "f32-bf16", "bf16-f32"])
@pytest.mark.parametrize("place", PLACES, ids=["whole", "part"])
def test_dropout(shape, layout, types, place):
    """The mask to the bit, one product and one rounding; nothing beside the tensor touched."""
    tx, ty = types.split("-")
    x, _ = put(layout, randn(rng(1), *shape), tx)
    y, mem = A.tensor(layout, *shape, ty)
    p, seed = 0.3, 2 ** 64 - 5
    dc.dropout(dc.Drop(p, seed, **place), V(x), x, V(y), y)
    m = R.mask(shape, p, seed, **place, device="cuda")
    want = f64(x) * m
    near(y, want, 2 * R.EPS32 * want.abs(), "y")
    assert torch.equal(f64(y) == 0, (m == 0) | (f64(x) == 0))
    assert A.untouched(y, mem)


# 16 bytes a thread: 2048 waves and more; eights of channels in two workgroups' widths
DROP_SIZES = [((2, 64, 150, 151), "dense"), ((1, 100, 213, 211), "gaps"), ((3, 43, 200, 230), "padded"), ((40, 2500, 30, 1), "rows"),
              ((3, 520, 333, 1), "slice")]


@pytest.mark.parametrize("shape,layout", DROP_SIZES, ids=str)
@pytest.mark.parametrize("types", ["f32-f32", "bf16-bf16", "f32-bf16", "bf16-f32"])
def test_dropout_sizes(shape, layout, types):
    test_dropout(shape, layout, types, {"h0": 1, "w0": 2, "H": 1000, "W": 999})


def test_dropout_in_place_of_everything_and_nothing():
    g = rng(2)
    x = randn(g, 2, 20, 6, 9).cuda()
    x[0, 3], x[1, 7] = float("nan"), float("inf")
    for p in (0.0, 2.0 ** -17, 0.5, 1 - 2.0 ** -30):
        m = R.mask(x.shape, p, 9, device="cuda").view(x.shape)
        y = x.clone()
        dc.dropout(dc.Drop(p, 9), V(y), y, V(y), y)
        want = torch.where(m == 0, 0.0, x.double() * m)              # what is dropped is 0, whatever stood there
        assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y.isinf(), want.isinf())
        fine = torch.isfinite(want)
        assert bool(((y - want).abs()[fine] <= 2 * R.EPS32 * want.abs()[fine]).all())
        assert p != 0 or torch.equal(torch.nan_to_num(y), torch.nan_to_num(x))
    assert int((y != 0).sum()) <= 2 * 20 * 6 * 9 // 100


def test_dropout_of_tiles_is_that_of_the_whole_image():
    """All tiles of a 2 x 3 grid as samples, each tile alone, and the image."""
    P, Q, N, C, h, w = 2, 3, 2, 19, 5, 7
    x = randn(rng(3), N, C, P * h, Q * w).cuda()
    y = torch.empty_like(x)
    dc.dropout(dc.Drop(0.4, 77, 5), V(x), x, V(y), y)
    tiles = x.view(N, C, P, h, Q, w).permute(2, 4, 0, 1, 3, 5).reshape(P * Q * N, C, h, w).contiguous()
    out = torch.empty_like(tiles)
    dc.dropout(dc.Drop(0.4, 77, 5, P=P, Q=Q), V(tiles), tiles, V(out), out)
    back = out.view(P, Q, N, C, h, w).permute(2, 3, 0, 4, 1, 5).reshape(x.shape)
    assert torch.equal(back, y)
    one = torch.empty(1, C, h, w, device="cuda")
    for t in range(P * Q):
        p, q = divmod(t, Q)
        dc.dropout(dc.Drop(0.4, 77, 5, n0=1, h0=p * h, w0=q * w, H=P * h, W=Q * w), V(one), tiles[t * N + 1:t * N + 2], V(one), one)
        assert torch.equal(one[0], out[t * N + 1])


def test_dropout_of_rows_is_that_of_planes():
    x = randn(rng(4), 3, 100, 37, 1).to(torch.bfloat16).cuda()
    y = torch.empty_like(x)
    dc.dropout(dc.Drop(0.2, 1), V(x), x, V(y), y)
    r, _ = put("rows", x.float().cpu(), "bf16")
    z, _ = A.tensor("rows", 3, 100, 37, 1, "bf16")
    dc.dropout(dc.Drop(0.2, 1), V(r), r, V(z), z)
    assert torch.equal(y, z)


def test_dropout_positions_past_32_bits():
    """A part of a tensor of more than 2^32 eights of channels (2^55; past 2^63 the call is refused), and a
    view whose samples lie 2^31 elements apart."""
    place = {"n0": 2 ** 20 - 9, "h0": 70000, "w0": 80000, "H": 90000, "W": 90000}
    x = torch.ones(2, 33, 3, 11, device="cuda")
    y = torch.empty_like(x)
    dc.dropout(dc.Drop(0.5, 123, **place), V(x), x, V(y), y)
    assert torch.equal(f64(y), R.mask(x.shape, 0.5, 123, **place, device="cuda"))
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 9 GB of the card")
    mem = torch.zeros((1 << 31) + 2000, device="cuda")
    far = torch.as_strided(mem, (2, 33, 3, 11), (1 << 31, 33, 11, 1))
    far.fill_(1.0)
    dc.dropout(dc.Drop(0.5, 123, **place), V(far), far, V(far), far)
    assert torch.equal(far, y)


# ------------------------------------------------------------------ the gated product

def gate_case(g, shape, layout, dtype):
    N, C, H, W, K = shape
    x, _ = put(layout, randn(g, N, C, H, W), dtype)
    w = (randn(g, 2 * K, C) / C ** 0.5).to(A.DT[dtype]).cuda()
    return x, w, vec(g, 2 * K)


def kept_bound(z, e, keep, K):
    """Of what is kept: in 8 bits half a step of 2^-6 of the block's power of two (a whole one at its
    very top), and the power itself may round up."""
    if keep != "q8":
        return e
    N, _, P = z.shape
    full = torch.zeros(N, -(-K // 32) * 32, P, dtype=torch.float64, device=z.device)
    full[:, :K] = z.abs()
    power = torch.exp2(torch.floor(torch.log2(full.view(N, -1, 32, P).amax(2).clamp(min=2.0 ** -120))))
    return 2.0 ** -6 * power.repeat_interleave(32, 1)[:, :K] * (1 + 1e-5) + e


def check_gate(shape, layout, dtype, out, keep, act, p):
    N, C, H, W, K = shape
    g = rng(5)
    x, w, b = gate_case(g, shape, layout, dtype)
    place = {"n0": 1, "h0": 1, "w0": 2, "H": H + 3, "W": W + 4, "offset": 3}
    drop = dc.Drop(p, 11, **place) if p else None
    m = R.mask((N, K, H, W), p, 11, **place, device="cuda") if p else torch.ones(1, 1, 1, dtype=torch.float64, device="cuda")
    h, hmem = A.tensor(layout, N, K, H, W, out)
    vz, zg, zu = None, None, None
    if keep == "q8":
        vz, zg, zu = dc.View.q8(N, K, H, W), ckpt(N, K, H, W), ckpt(N, K, H, W)
    elif keep:
        (zg, gmem), (zu, umem) = A.tensor(layout, N, K, H, W, keep), A.tensor(layout, N, K, H, W, keep)
        vz = V(zg)
    dc.gate_fwd(V(x), x, w, b, dc.ACT[act], drop, vz, zg, zu, V(h), h)
    wg, wu, eg, eu = R.gate_sums(f64(x), w.double(), b.double())
    near(h, *R.gate(wg, wu, eg, eu, act, m), "h")
    assert A.untouched(h, hmem)
    if not keep:
        return
    ks = []
    for z, want, e in ((zg, wg, eg), (zu, wu, eu)):
        if keep == "q8":
            zs = decode(z, N, K, H, W)
            near(zs, want, kept_bound(want, e, keep, K), "z8")
        else:
            zs = f64(z)
            near(z, want, e, "z")
        ks.append(zs)
    assert keep == "q8" or (A.untouched(zg, gmem) and A.untouched(zu, umem))
    dy, _ = put(layout, randn(g, N, C, H, W), dtype)
    w2 = (randn(g, C, K) / K ** 0.5).to(A.DT[dtype]).cuda()
    dz, dmem = A.tensor(layout, N, 2 * K, H, W, out)
    h.fill_(float("nan"))
    dc.gate_bwd_data(V(dy), dy, w2, dc.ACT[act], drop, vz, zg, zu, V(h), h, V(dz), dz)
    dg, du, wh, bg, bu, bh = R.gate_bwd(f64(dy), w2.double(), *ks, act, m)
    near(dz[:, :K], dg, bg, "dzg")
    near(dz[:, K:], du, bu, "dzu")
    near(h, wh, bh, "h again")
    assert A.untouched(dz, dmem) and A.untouched(h, hmem)
    again = torch.empty_like(dz)
    dc.gate_bwd_data(V(dy), dy, w2, dc.ACT[act], drop, vz, zg, zu, None, None, V(again), again)
    assert torch.equal(again, dz)


GATE_TYPES = [("f32", "f32", "f32", "gelu", 0.0), ("bf16", "bf16", "q8", "silu", 0.25), ("bf16", "f32", "bf16", "none", 0.0),
              ("f32", "bf16", "q8", "relu", 0.6), ("bf16", "bf16", None, "gelu", 0.1), ("f32", "f32", "bf16", "silu", 0.3)]


@pytest.mark.parametrize("shape,layout", T.PLAYOUTS, ids=str)
@pytest.mark.parametrize("types", GATE_TYPES, ids=str)
def test_gate(shape, layout, types):
    check_gate(shape, layout, *types)


# every block that the sizes pick: large, middle, short, few pixels with long sums; whole and ragged, planes and rows
GATE_BLOCKS = {
    "large": ((2, 136, 130, 132, 256), "dense"), "large_ragged": ((1, 257, 181, 183, 259), "gaps"),
    "large_rows": ((9, 264, 3700, 1, 264), "rows"), "large_slice": ((33000, 263, 1, 1, 261), "slice"),
    "middle": ((1, 128, 150, 304, 136), "dense"), "middle_off": ((1, 100, 151, 301, 133), "dense"), "middle_rows": ((35, 128, 1000, 1, 136), "slice"),
    "short": ((2, 32, 200, 250, 72), "padded"), "short_off": ((1, 24, 201, 251, 40), "gaps"), "short_rows": ((33000, 32, 1, 1, 136), "rows"),
    "few_long": ((2, 300, 23, 29, 70), "dense"), "few_long_rows": ((700, 263, 1, 1, 40), "slice"),
}


@pytest.mark.parametrize("name", GATE_BLOCKS)
@pytest.mark.parametrize("types", GATE_TYPES[:2], ids=str)
def test_gate_blocks(name, types):
    check_gate(*GATE_BLOCKS[name], *types)


# up to 16 pixels of many channels: k that ends with a whole group of steps, a step, part of one, and that one group holds
GATE_FEW = [((1, 1000, 1, 1, 4104), "rows"), ((3, 200, 2, 2, 4100), "dense"), ((16, 70, 1, 1, 4099), "slice"), ((7, 2048, 1, 1, 4096), "rows"),
            ((1, 31, 3, 5, 4111), "gaps"), ((33, 1056, 1, 1, 72), "rows"), ((1, 1, 1, 1, 4096), "rows"), ((50, 96, 1, 1, 1), "rows")]


@pytest.mark.parametrize("shape,layout", GATE_FEW, ids=str)
@pytest.mark.parametrize("types", GATE_TYPES, ids=str)
def test_gate_few(shape, layout, types):
    check_gate(shape, layout, *types)


def test_gate_without_bias_in_mixed_layouts():
    g = rng(6)
    for lx, lh in (("rows", "dense"), ("dense", "rows"), ("slice", "gaps")):
        x, w, _ = gate_case(g, (3, 40, 30, 1, 50), lx, "bf16")
        h, mem = A.tensor(lh, 3, 50, 30, 1, "f32")
        dc.gate_fwd(V(x), x, w, None, dc.DC_ACT_SILU, None, None, None, None, V(h), h)
        zg, zu, eg, eu = R.gate_sums(f64(x), w.double(), torch.zeros(100, dtype=torch.float64, device="cuda"))
        near(h, *R.gate(zg, zu, eg, eu, "silu", 1.0), "h")
        assert A.untouched(h, mem)


@pytest.mark.parametrize("path", ["few", "small", "rows"])
def test_gate_keeps_what_is_not_finite_to_its_pixel(path):
    N, C, H, W, layout = {"few": (1, 70, 6, 9, "dense"), "small": (2, 70, 20, 21, "dense"), "rows": (300, 72, 1, 1, "rows")}[path]
    g = rng(7)
    v = randn(g, N, C, H, W)
    v[0, 5, 0, 0], v[N - 1, 66, H - 1, W - 1] = float("inf"), float("nan")
    x, _ = put(layout, v, "bf16")
    w = randn(g, 80, C).to(torch.bfloat16).cuda()
    h = torch.empty(N, 40, H, W, device="cuda")
    dc.gate_fwd(V(x), x, w, None, dc.DC_ACT_RELU, None, None, None, None, V(h), h)
    zg, zu, _, _ = R.gate_sums(f64(x), w.double(), torch.zeros(80, dtype=torch.float64, device="cuda"))
    want = R.act(zg, "relu") * zu
    got = f64(h)
    assert torch.equal(torch.isfinite(got).all(1), torch.isfinite(want).all(1))
    assert torch.equal(torch.isnan(got), torch.isnan(want))


# ------------------------------------------------------------------ the join

# y, x, o, u and gradients' types; norms; scale, gate, dropout; what the backward pass reads in 8 bits
JOINS = {
    "all": dict(types="f32-f32-f32-f32", post="layer", pre="layer", scale=True, gate=True, p=0.25),
    "rms": dict(types="bf16-f32-f32-bf16", post="rms", pre="rms", scale=True, q8=True),
    "gate": dict(types="f32-bf16-bf16-f32", pre="layer", gate=True, p=0.6),
    "post": dict(types="bf16-bf16-bf16-bf16", post="rms", scale=True, p=0.1),
    "mixed": dict(types="bf16-f32-bf16-bf16", post="layer", pre="rms", gate=True, scale=True, p=0.1, q8=True),
    "plain": dict(types="f32-f32-f32-f32"),
}


def check_join(shape, layout, types, post=None, pre=None, scale=False, gate=False, p=0.0, q8=False):
    ty, tx, to, tu = types.split("-")
    N, C, H, W = shape
    g = rng(8)
    y, _ = put(layout, 0.7 * randn(g, *shape) + randn(g, 1, C, 1, 1), ty)
    x, _ = put(layout, randn(g, *shape) + randn(g, 1, C, 1, 1), tx)
    par = {k: vec(g, C, mean=float(k[0] == "g")) for k in ("gamma_post", "beta_post", "gamma_pre", "beta_pre")}
    sc, gt = (vec(g, C, mean=0.5) if scale else None), (vec(g, N, C, mean=1.0) if gate else None)
    place = {"n0": 2, "h0": 3, "w0": 1, "H": H + 5, "W": W + 2, "offset": 7}
    drop = dc.Drop(p, 2 ** 60 + 1, **place) if p else None
    m = R.mask(shape, p, 2 ** 60 + 1, **place, device="cuda") if p else torch.ones(N, C, H * W, dtype=torch.float64, device="cuda")
    n = {k: dc.Norm(dc.NORM[v], EPS, par["gamma_" + k], par["beta_" + k]) if v else None for k, v in (("post", post), ("pre", pre))}
    (o, omem), (u, umem) = A.tensor(layout, *shape, to), A.tensor(layout, *shape, tu)
    stat = torch.full((4, N, H, W), float("nan"), device="cuda")
    q = ckpt(*shape) if q8 else None
    vu, pu = (V(u), u) if pre else (None, None)
    dc.join_fwd(V(y), y, n["post"], sc, gt, drop, V(x), x, n["pre"], V(o), o, vu, pu, stat, q)
    d = {k: v.double() for k, v in par.items()}
    one = torch.ones(1, dtype=torch.float64, device="cuda")
    s64 = sc.double() if scale else one.expand(C)
    g64 = gt.double() if gate else one.expand(N, C)
    rp = (post, d["gamma_post"], d["beta_post"]) if post else None
    rq = (pre, d["gamma_pre"], d["beta_pre"]) if pre else None
    want = R.join(f64(y), rp, (s64 * g64)[:, :, None], m, f64(x), rq, EPS)
    near(o, *want["o"], "o")
    assert A.untouched(o, omem)
    if pre:
        near(u, *want["u"], "u")
        assert A.untouched(u, umem)
    st = stat.double().view(2, 2, N, 1, H * W)
    for k, name, on in ((0, "stat", post), (1, "stat2", pre)):
        if on:
            for i, w in enumerate(want[name]):
                near(st[k, i], *w, name)
        else:
            assert bool(torch.isnan(stat[2 * k:2 * k + 2]).all())
    if q8:
        near(decode(q, *shape), want["o"][0], kept_bound(want["o"][0], want["o"][1], "q8", C), "o in 8 bits")
    # backward
    du, _ = put(layout, randn(g, *shape), tu)
    dr, _ = put(layout, randn(g, *shape), to)
    (dx, xmem), (dy, ymem) = A.tensor(layout, *shape, to), A.tensor(layout, *shape, ty)
    vo, po, o64 = V(o), o, f64(o)
    vy, py, y64 = V(y), y, f64(y)
    vx, px, x64 = V(x), x, f64(x)
    if q8:
        yq, xq = ckpt(*shape), ckpt(*shape)
        dc.ckpt_save(V(y), y, yq)
        dc.ckpt_save(V(x), x, xq)
        vo = vy = vx = dc.View.q8(*shape)
        po, o64, py, y64, px, x64 = q, decode(q, *shape), yq, decode(yq, *shape), xq, decode(xq, *shape)
    st = [(st[k, 0], st[k, 1]) for k in range(2)]
    need = dc.join_bwd_workspace_bytes(V(dy), gate)
    # dgate is wanted without dscale now and then, and the other way
    grads = {"scale": vec(g, C), "gate": vec(g, N, C) if gate else None, **{k + "_post": vec(g, C) if post else None for k in ("gamma", "beta")},
             **{k + "_pre": vec(g, C) if pre else None for k in ("gamma", "beta")}}
    before = {k: t.double().clone() for k, t in grads.items() if t is not None}
    vdu, pdu = (V(du), du) if pre else (None, None)
    args = (vdu, pdu, V(dr), dr, vy, py, None, None, vo, po, stat, n["post"], sc, gt, drop, n["pre"])
    dc.join_bwd(*args, V(dx), dx, V(dy), dy, dc.JoinGrads(**grads), 1, ws(need))
    want = R.join_bwd(f64(du) if pre else None, f64(dr), y64, o64, st, rp, s64, g64, m, rq)
    near(dx, *want["dx"], "dx")
    near(dy, *want["dy"], "dy")
    for k, b in before.items():
        near(grads[k], b + want[k][0], want[k][1] + 2 * R.EPS32 * (b + want[k][0]).abs(), "d" + k)
    assert A.untouched(dx, xmem) and A.untouched(dy, ymem)
    # overwriting some, without the residual's; the rest to the bit; then without any gradient
    over = {k: torch.full_like(t, float("nan")) for k, t in grads.items() if t is not None and k in ("gate", "gamma_pre", "beta_post")}
    dy2 = torch.empty_like(dy)
    dc.join_bwd(*args, None, None, V(dy2), dy2, dc.JoinGrads(**over), 0, ws(need))
    assert torch.equal(dy2, dy)
    for k, t in over.items():
        near(t, *want[k], "d" + k)
    dy2.fill_(0)
    dc.join_bwd(*args, None, None, V(dy2), dy2, None, 0, None)
    assert torch.equal(dy2, dy)
    if pre:          # o formed again from y and x, as the backward pass has them
        v64 = d["gamma_post"][:, None] * (y64 - st[0][0]) * st[0][1] + d["beta_post"][:, None] if post else y64
        ev = 4 * R.EPS32 * (v64.abs() + d["beta_post"].abs()[:, None]) + \
            (3 * R.EPS32 * d["gamma_post"].abs()[:, None] * st[0][1] * (y64.abs() + st[0][0].abs()) if post else 0)
        f = (s64 * g64)[:, :, None] * m
        formed = x64 + f * v64
        eo = f.abs() * ev + 4 * R.EPS32 * (f * v64).abs() + 2 * R.EPS32 * formed.abs()
        for t in grads.values():
            if t is not None:
                t.fill_(float("nan"))
        dc.join_bwd(*args[:6], vx, px, None, None, *args[10:], V(dx), dx, V(dy), dy, dc.JoinGrads(**grads), 0, ws(need))
        want = R.join_bwd(f64(du), f64(dr), y64, formed, st, rp, s64, g64, m, rq, eo)
        near(dx, *want["dx"], "dx formed")
        near(dy, *want["dy"], "dy formed")
        for k in before:
            near(grads[k], *want[k], "formed d" + k)
    if pre:          # without what is read at o elsewhere
        dc.join_bwd(*args[:2], None, None, *args[4:], V(dx), dx, V(dy2), dy2, None, 0, None)
        want = R.join_bwd(f64(du), None, y64, o64, st, rp, s64, g64, m, rq)
        near(dx, *want["dx"], "dx")
        near(dy2, *want["dy"], "dy")


@pytest.mark.parametrize("shape,layout", T.LAYOUTS, ids=str)
@pytest.mark.parametrize("name", JOINS)
def test_join(shape, layout, name):
    check_join(shape, layout, **JOINS[name])


# whole tiles (64 pixels a wave) with one and two blocks a lane, many turns and samples, rows and tiles of too many
# channels for the registers, gates of a sample a row and of more samples than walkers
JOIN_SIZES = [((1, 40, 300, 231), "gaps"), ((3, 64, 160, 161), "dense"), ((2, 300, 121, 61), "padded"), ((1, 512, 120, 101), "dense"),
              ((5, 24, 209, 111), "dense"), ((1100, 40, 3, 2), "dense"), ((3000, 100, 1, 1), "rows"), ((37, 520, 45, 1), "slice"),
              ((5, 4104, 40, 1), "rows"), ((2, 1056, 30, 33), "dense"), ((2500, 1, 1, 1), "rows"), ((3, 8200, 21, 1), "rows"),
              ((2, 8999, 4, 1), "slice"), ((2, 2300, 9, 40), "dense"), ((4, 20, 60, 61), "gaps")]


@pytest.mark.parametrize("shape,layout", JOIN_SIZES, ids=str)
@pytest.mark.parametrize("name", ["all", "rms", "mixed"])
def test_join_sizes(shape, layout, name):
    check_join(shape, layout, **JOINS[name])


def test_join_in_place_and_without_a_residual():
    """o over x, u over y, dx over d_o, dy over y, to the bit; no x is an x of zeros."""
    g = rng(9)
    for shape, layout in (((2, 48, 9, 11), "dense"), ((3, 600, 7, 1), "rows"), ((1, 4200, 5, 1), "rows"), ((1, 1100, 4, 5), "dense"),
                          ((2, 8300, 3, 1), "rows"), ((1, 2100, 4, 5), "gaps"), ((2, 20, 33, 35), "dense"), ((3, 200, 40, 41), "padded")):
        N, C, H, W = shape
        y, _ = put(layout, randn(g, *shape), "f32")
        x, _ = put(layout, randn(g, *shape), "f32")
        post, pre = dc.Norm(dc.DC_NORM_LAYER, EPS, vec(g, C, mean=1.0)), dc.Norm(dc.DC_NORM_RMS, EPS, None, vec(g, C))
        drop, stat = dc.Drop(0.2, 5), torch.empty(4, N, H, W, device="cuda")
        o, u = torch.empty_like(x), torch.empty_like(x)
        dc.join_fwd(V(y), y, post, None, None, drop, V(x), x, pre, V(o), o, V(u), u, stat)
        ox, uy, y2 = x.clone(), y.clone(), y.clone()
        dc.join_fwd(V(uy), uy, post, None, None, drop, V(ox), ox, pre, V(ox), ox, V(uy), uy)
        assert torch.equal(ox, o) and torch.equal(uy, u)
        du, dr = torch.randn_like(u), torch.randn_like(o)
        dx, dy = torch.empty_like(x), torch.empty_like(x)
        dc.join_bwd(V(du), du, V(dr), dr, V(y), y, None, None, V(o), o, stat, post, None, None, drop, pre, V(dx), dx, V(dy), dy, None, 0, None)
        dc.join_bwd(V(du), du, V(dr), dr, V(y2), y2, None, None, V(o), o, stat, post, None, None, drop, pre, V(dr), dr, V(y2), y2, None, 0, None)
        assert torch.equal(dr, dx) and torch.equal(y2, dy)
        dc.join_fwd(V(y), y, post, None, None, drop, None, None, pre, V(o), o, V(u), u)
        zero = torch.zeros_like(x)
        dc.join_fwd(V(y), y, post, None, None, drop, V(zero), zero, pre, V(ox), ox, V(uy), uy)
        assert torch.equal(o, ox) and torch.equal(u, uy)


def test_join_of_constant_and_offset_pixels():
    """No variance: u = beta where the mean is exact; a mean of 2^12 spreads costs what the input's own
    24 bits allow; a row of zeros under the root mean square stays zero."""
    x = torch.full((1, 64, 1, 4), 0.5)
    x[0, :, 0, 1] = 0.0
    x[0, :, 0, 2] = 4096 + randn(rng(10), 64)
    t, beta, zero = x.cuda(), vec(rng(11), 64), torch.zeros(1, 64, 1, 4, device="cuda")
    o, u = torch.empty_like(t), torch.empty_like(t)
    dc.join_fwd(V(zero), zero, None, None, None, None, V(t), t, dc.Norm(dc.DC_NORM_LAYER, EPS, None, beta), V(o), o, V(u), u)
    assert torch.equal(o, t)
    for k in (0, 1):
        assert torch.equal(u[0, :, 0, k], beta)
    one = torch.ones(64, dtype=torch.float64, device="cuda")
    want, mu, r = R.norm(f64(t), "layer", one, beta.double(), EPS)
    near(u, want, R.norm_tol(f64(t), mu, r, one, beta.double()), "u")
    dc.join_fwd(V(zero), zero, None, None, None, None, V(t), t, dc.Norm(dc.DC_NORM_RMS, EPS), V(o), o, V(u), u)
    assert not bool(u[0, :, 0, 1].any())


def test_join_keeps_what_is_not_finite_to_its_pixel():
    """And what is dropped out stays out: a NaN in a dropped place reaches nothing."""
    g = rng(12)
    for layout, shape in (("dense", (1, 70, 4, 33)), ("rows", (2, 70, 66, 1))):
        N, C, H, W = shape
        v = randn(g, *shape)
        drop = dc.Drop(0.5, 3)
        m = R.mask(shape, 0.5, 3).view(shape)
        gone = (m == 0).nonzero()[5].tolist()
        stays = (m != 0).nonzero()[-9].tolist()
        v[tuple(gone)], v[tuple(stays)] = float("nan"), float("inf")
        y, _ = put(layout, v, "f32")
        x, _ = put(layout, randn(g, *shape), "f32")
        o, u, stat = torch.empty_like(x), torch.empty_like(x), torch.empty(4, N, H, W, device="cuda")
        pre = dc.Norm(dc.DC_NORM_LAYER, EPS)
        dc.join_fwd(V(y), y, None, None, None, drop, V(x), x, pre, V(o), o, V(u), u, stat)
        bad = torch.zeros(N, H, W, dtype=torch.bool)
        bad[stays[0], stays[2], stays[3]] = True
        assert torch.equal((~torch.isfinite(o)).any(1).cpu(), bad) and torch.equal((~torch.isfinite(u)).all(1).cpu(), bad)
        assert int((~torch.isfinite(o)).sum()) == 1
        du, dx, dy = torch.randn_like(u), torch.empty_like(x), torch.empty_like(x)
        dc.join_bwd(V(du), du, None, None, None, None, None, None, V(o), o, stat, None, None, None, drop, pre, V(dx), dx, V(dy), dy, None, 0, None)
        assert torch.equal(torch.isfinite(dx).all(1).cpu(), ~bad)
        assert not bool(torch.where(m.cuda() == 0, dy, torch.zeros_like(dy)).any())       # also where dx is NaN


def test_join_broadcast_inputs():
    """Strides of 0 in what is read: one branch and one gradient for every sample and row."""
    g = rng(13)
    y = randn(g, 1, 40, 1, 9).cuda().expand(3, 40, 5, 9)
    x = randn(g, 3, 40, 5, 9).cuda()
    o, u, stat = torch.empty_like(x), torch.empty_like(x), torch.empty(4, 3, 5, 9, device="cuda")
    one, zero = torch.ones(40, dtype=torch.float64, device="cuda"), torch.zeros(40, dtype=torch.float64, device="cuda")
    n = dc.Norm(dc.DC_NORM_LAYER, EPS)
    dc.join_fwd(V(y), y, n, None, None, None, V(x), x, n, V(o), o, V(u), u, stat)
    m = torch.ones(3, 40, 45, dtype=torch.float64, device="cuda")
    want = R.join(f64(y.contiguous()), ("layer", one, zero), torch.ones(3, 40, 1, dtype=torch.float64, device="cuda"), m, f64(x),
                  ("layer", one, zero), EPS)
    near(o, *want["o"], "o")
    near(u, *want["u"], "u")
    du = randn(g, 1, 40, 1, 9).cuda().expand(3, 40, 5, 9)
    dx, dy = torch.empty_like(x), torch.empty_like(x)
    dc.join_bwd(V(du), du, None, None, V(y), y, None, None, V(o), o, stat, n, None, None, None, n, V(dx), dx, V(dy), dy, None, 0, None)
    st = [(stat[2 * k].double().view(3, 1, 45), stat[2 * k + 1].double().view(3, 1, 45)) for k in range(2)]
    want = R.join_bwd(f64(du.contiguous()), None, f64(y.contiguous()), f64(o), st, ("layer", one, zero), one, one.expand(3, 40), m,
                      ("layer", one, zero))
    near(dx, *want["dx"], "dx")
    near(dy, *want["dy"], "dy")


def test_offsets_past_32_bits():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 36 GB of the card")
    g = rng(14)
    far, shape = 1 << 31, (2, 40, 6, 20)

    def tensor(C):
        mem = torch.empty(far + (1 << 18), device="cuda")
        return torch.as_strided(mem, (2, C, 6, 20), (far, 120, 20, 1))

    y, x, o, u = (tensor(40) for _ in range(4))
    y.copy_(randn(g, *shape))
    x.copy_(randn(g, *shape))
    n, stat = dc.Norm(dc.DC_NORM_LAYER, EPS), torch.empty(4, 2, 6, 20, device="cuda")
    dc.join_fwd(V(y), y, n, None, None, None, V(x), x, n, V(o), o, V(u), u, stat)
    c = [t.contiguous() for t in (y, x)]
    oc, uc = torch.empty_like(c[0]), torch.empty_like(c[0])
    dc.join_fwd(V(c[0]), c[0], n, None, None, None, V(c[1]), c[1], n, V(oc), oc, V(uc), uc)
    assert torch.equal(o, oc) and torch.equal(u, uc)
    w, hc = randn(g, 60, 40).cuda(), torch.empty(2, 30, 6, 20, device="cuda")
    h = torch.as_strided(y, (2, 30, 6, 20), (far, 120, 20, 1))
    dc.gate_fwd(V(u), u, w, None, dc.DC_ACT_GELU, None, None, None, None, V(h), h)
    dc.gate_fwd(V(uc), uc, w, None, dc.DC_ACT_GELU, None, None, None, None, V(hc), hc)
    assert torch.equal(h, hc)


# ------------------------------------------------------------------ together, streams and graphs

class Block:
    """A gated residual block as a program runs it: norm, gated product, product, join; trained."""

    def __init__(self, seed, N=2, C=48, H=13, W=30, F=72, dtype=torch.bfloat16, step=None):
        g = rng(seed)
        self.shape = N, C, H, W
        self.F, bf = F, dtype
        self.x = randn(g, N, C, H, W).cuda()
        self.w1, self.w2 = (randn(g, 2 * F, C) / C ** 0.5).to(bf).cuda(), (randn(g, C, F) / F ** 0.5).to(bf).cuda()
        self.b1, self.b2 = vec(g, 2 * F), vec(g, C)
        self.p = {k: vec(g, C, mean=float(k[0] == "g")) for k in ("gamma0", "beta0", "gamma1", "beta1", "gamma2", "beta2")}
        self.scale, self.gate = vec(g, C, mean=0.5), vec(g, N, C, mean=1.0)
        self.hidden, self.out = dc.Drop(0.1, seed, 0, step=step), dc.Drop(0.2, seed, 1 << 32, step=step)
        self.post, self.pre = (dc.Norm(k, EPS, self.p["gamma" + i], self.p["beta" + i]) for k, i in ((dc.DC_NORM_RMS, "1"), (dc.DC_NORM_LAYER, "2")))
        e = lambda c, d=bf: torch.empty(N, c, H, W, dtype=d, device="cuda")   # noqa: E731
        f = lambda *s: torch.empty(*s, device="cuda")   # noqa: E731
        self.u, self.h, self.y, self.u2, self.dh = e(C), e(F), e(C), e(C), e(F)
        self.o, self.dr, self.dx = e(C, torch.float32), e(C, torch.float32), e(C, torch.float32)
        self.dy, self.du, self.dz = e(C), e(C), e(2 * F)
        self.du2 = randn(g, N, C, H, W).to(bf).cuda()
        self.dr.copy_(randn(g, N, C, H, W))
        self.stat0, self.stat = f(2, N, H, W), f(4, N, H, W)
        self.q = dc.View.q8(N, F, H, W)
        self.zg, self.zu = ckpt(N, F, H, W), ckpt(N, F, H, W)
        self.grads = dc.JoinGrads(f(C), f(N, C), f(C), f(C), f(C), f(C))
        self.dw1, self.db1, self.dw2, self.db2, self.dg0, self.db0 = f(2 * F, C), f(2 * F), f(C, F), f(C), f(C), f(C)
        self.ws = ws(max(dc.join_bwd_workspace_bytes(V(self.dy), True), dc.norm_bwd_workspace_bytes(V(self.du)),
                         dc.linear_bwd_filter_workspace_bytes(V(self.u), V(self.dz)),
                         dc.linear_bwd_filter_workspace_bytes(V(self.h), V(self.dy))))

    def step(self):
        s, p = self, self.p
        dc.norm_fwd(V(s.x), s.x, p["gamma0"], p["beta0"], EPS, V(s.u), s.u, s.stat0)
        dc.gate_fwd(V(s.u), s.u, s.w1, s.b1, dc.DC_ACT_SILU, s.hidden, s.q, s.zg, s.zu, V(s.h), s.h)
        dc.linear_fwd(V(s.h), s.h, s.w2, s.b2, dc.DC_ACT_NONE, None, None, None, None, V(s.y), s.y)
        dc.join_fwd(V(s.y), s.y, s.post, s.scale, s.gate, s.out, V(s.x), s.x, s.pre, V(s.o), s.o, V(s.u2), s.u2, s.stat)
        dc.join_bwd(V(s.du2), s.du2, V(s.dr), s.dr, V(s.y), s.y, V(s.x), s.x, None, None, s.stat, s.post, s.scale, s.gate, s.out, s.pre,
                    V(s.dx), s.dx, V(s.dy), s.dy, s.grads, 0, s.ws)
        dc.gate_bwd_data(V(s.dy), s.dy, s.w2, dc.DC_ACT_SILU, s.hidden, s.q, s.zg, s.zu, V(s.dh), s.dh, V(s.dz), s.dz)
        dc.linear_bwd_filter(V(s.dh), s.dh, V(s.dy), s.dy, s.dw2, s.db2, 0, s.ws)
        dc.linear_bwd_data(V(s.dz), s.dz, s.w1, dc.DC_ACT_NONE, None, None, None, None, V(s.du), s.du)
        dc.linear_bwd_filter(V(s.u), s.u, V(s.dz), s.dz, s.dw1, s.db1, 0, s.ws)
        dc.norm_bwd(V(s.du), s.du, V(s.x), s.x, s.stat0, p["gamma0"], p["beta0"], V(s.dx), s.dx, None, None, V(s.dx), s.dx, s.dg0, s.db0,
                    0, s.ws)

    def results(self):
        g = self.grads
        return {"o": self.o, "u2": self.u2, "dx": self.dx, "dw1": self.dw1, "db1": self.db1, "dw2": self.dw2, "db2": self.db2, "dgamma0": self.dg0,
                "dbeta0": self.db0, "dscale": g.scale, "dgate": g.gate, "dgamma1": g.gamma_post, "dbeta1": g.beta_post, "dgamma2": g.gamma_pre,
                "dbeta2": g.beta_pre}

    def reference(self, step=0):
        """Automatic differentiation of the same block in 64 bits on the CPU."""
        N, C, H, W = self.shape
        leaf = {"x": self.x, "w1": self.w1, "b1": self.b1, "w2": self.w2, "b2": self.b2, "scale": self.scale, "gate": self.gate, **self.p}
        t = {k: v.detach().cpu().double().requires_grad_() for k, v in leaf.items()}
        mh = R.mask((N, self.F, H, W), 0.1, self.hidden.seed, 0, step)
        mo = R.mask((N, C, H, W), 0.2, self.out.seed, 1 << 32, step)
        x = t["x"].reshape(N, C, -1)
        u = R.norm(x, "layer", t["gamma0"], t["beta0"], EPS)[0]
        z = R.product(t["w1"], u) + t["b1"][:, None]
        h = torch.nn.functional.silu(z[:, :self.F]) * z[:, self.F:] * mh
        y = R.product(t["w2"], h) + t["b2"][:, None]
        o = x + (t["scale"] * t["gate"])[:, :, None] * mo * R.norm(y, "rms", t["gamma1"], t["beta1"], EPS)[0]
        u2 = R.norm(o, "layer", t["gamma2"], t["beta2"], EPS)[0]
        ((o * self.dr.cpu().double().reshape(o.shape)).sum() + (u2 * self.du2.cpu().double().reshape(o.shape)).sum()).backward()
        out = {"d" + k: v.grad for k, v in t.items()}
        out["o"], out["u2"] = o.detach().view(self.shape), u2.detach().view(self.shape)
        return out


def test_a_block_of_them_against_automatic_differentiation():
    """Each tensor in between is rounded to 8 significant bits a few times and the two sums kept for the
    backward pass to 7: relative errors of 2^-8 and 2^-7 at most, which average out over a gradient's
    sum.  The error over the length stays below 2^-5; a term left out or taken twice would be of order one."""
    for step in (None, 3):
        cell = None if step is None else torch.tensor([step], device="cuda")
        b = Block(15, step=cell)
        b.step()
        want = b.reference(step or 0)
        for k, got in b.results().items():
            w = want[k]
            err = float((got.cpu().double() - w).norm() / w.norm())
            assert err < 2 ** -5, (k, err)


def test_a_block_of_them_on_another_stream_and_in_graphs():
    """The same bits on a side stream and in every replay; two graphs that share a workspace; replays
    that draw new masks as the program counts the step up; eager work in between."""
    cell = torch.zeros(1, dtype=torch.int64, device="cuda")
    a, b = Block(16, step=cell), Block(17, N=3, C=40, F=100, step=cell)
    a.ws = b.ws = ws(max(a.ws.numel(), b.ws.numel()))

    def eager(s, step):
        cell.fill_(step)
        s.step()
        torch.cuda.synchronize()
        return {k: t.clone() for k, t in s.results().items()}

    want = {(s, k): eager(s, k) for s in (a, b) for k in range(3)}
    assert not torch.equal(want[a, 0]["o"], want[a, 1]["o"])
    side = torch.cuda.Stream()
    cell.fill_(1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    side.synchronize()
    assert all(torch.equal(t, want[a, 1][k]) for k, t in a.results().items())
    graphs = {}
    for s in (a, b):
        graphs[s] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[s]):
            s.step()
    for k in (0, 2, 1, 0):
        cell.fill_(k)
        for s in (a, b):
            for t in s.results().values():
                t.fill_(0)
            graphs[s].replay()
        torch.cuda.synchronize()
        for s in (a, b):
            for n, t in s.results().items():
                assert torch.equal(t, want[s, k][n]), (n, k)
        eager(a, 2)
