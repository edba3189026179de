"""Host-side checks of a gated residual block's operators: refusals before any launch, and the
oracles of the GPU tests (the generator's published vectors, gradients against automatic
differentiation and differences).  No GPU."""
import ctypes

import numpy as np
import pytest
import torch

import act_ref as A
import block_ref as R
import paper_1903_06681_amd as dc
from test_act_host import MIS2, MIS16, Ws, status, view

P1, P2, P3, P4 = 0x10000, 0x20000, 0x30000, 0x40000


def with_(fn, base):
    return lambda **kw: status(fn, *{**base, **kw}.values())


# ------------------------------------------------------------------ refusals

BAD_DROPS = [({"p": -0.1}, -10), ({"p": 1.0}, -10), ({"p": float("nan")}, -10), ({"n0": -1}, -10), ({"h0": -1}, -10), ({"w0": -1}, -10),
             ({"H": -1}, -10), ({"P": -1}, -10), ({"Q": -2}, -10), ({"P": 3}, -2), ({"H": 3}, -2), ({"W": 5}, -2), ({"h0": 1, "H": 4}, -2),
             ({"P": 2, "H": 7}, -2), ({"Q": 2, "W": 11}, -2), ({"step": 0x10004}, -7), ({"H": 2 ** 31 - 1, "W": 2 ** 31 - 1, "n0": 9}, -11)]


@pytest.mark.parametrize("kw,code", BAD_DROPS, ids=str)
def test_bad_drops(kw, code):
    d, v = dc.Drop(**{"p": 0.1, "seed": 1, **kw}), view()
    vz = view(C=16)
    assert status(dc.dropout, d, v, P1, v, P2, 0) == code
    assert status(dc.gate_fwd, v, P1, P2, None, 0, d, None, None, None, v, P3, 0) == code
    assert status(dc.gate_bwd_data, v, P1, P2, 0, d, v, P3, P4, None, None, vz, P3, 0) == code
    assert status(dc.join_fwd, v, P1, None, None, None, d, None, None, None, v, P2, None, None, None, None, 0) == code
    assert status(dc.join_bwd, None, None, v, P1, None, None, None, None, None, None, None, None, None, None, d, None, None, None, v, P2,
                  None, 0, None, 0) == code


def test_dropout_refusals():
    v, d = view(), dc.Drop(0.5, 1)
    call = with_(dc.dropout, dict(drop=d, vx=v, x=P1, vy=v, y=P2, stream=0))
    assert call(drop=None) == -1 and call(vx=None) == -1 and call(x=None) == -1 and call(vy=None) == -1 and call(y=None) == -1
    assert call(vy=view(C=9)) == -2 and call(vx=dc.View.q8(2, 8, 4, 6)) == -3 and call(vy=view(sc=23)) == -2
    assert call(x=MIS2) == -7 and call(y=MIS2) == -7


def test_gate_refusals():
    vx, vh, vz2 = view(), view(C=12), view(C=24)
    q = dc.View.q8(2, 12, 4, 6)
    call = with_(dc.gate_fwd, dict(vx=vx, x=P1, w=P2, bias=None, act=2, drop=None, vz=None, zg=None, zu=None, vh=vh, h=P3, stream=0))
    assert call(vx=None) == -1 and call(x=None) == -1 and call(w=None) == -1 and call(vh=None) == -1 and call(h=None) == -1
    assert call(act=-1) == -10 and call(act=4) == -10 and call(w=MIS16) == -7 and call(bias=MIS16) == -7
    assert call(vh=view(C=12, H=3)) == -2 and call(vh=q) == -3 and call(vh=view(C=12, sc=23)) == -2
    # both kept sums or none, in a view of K channels
    assert call(vz=vh, zg=P4) == -1 and call(vz=vh, zu=P4) == -1 and call(zg=P4, zu=P4) == -1 and call(vz=vx, zg=P4, zu=P4) == -2
    assert call(vz=q, zg=MIS16, zu=P4) == -7 and call(vz=q, zg=P4, zu=MIS16) == -7
    big = view(N=1, H=1, W=1, C=1 << 15)
    assert call(vx=big, vh=view(N=1, H=1, W=1, C=1 << 15)) == -11      # 2 K C = 2^31
    bwd = with_(dc.gate_bwd_data, dict(vdy=vx, dy=P1, w=P2, act=2, drop=None, vz=vh, zg=P3, zu=P4, vh=None, h=None, vdz=vz2, dz=P3,
                                       stream=0))
    assert bwd(vdy=None) == -1 and bwd(dy=None) == -1 and bwd(w=None) == -1 and bwd(vz=None) == -1 and bwd(zg=None) == -1
    assert bwd(zu=None) == -1 and bwd(vdz=None) == -1 and bwd(dz=None) == -1 and bwd(vh=None, h=P4) == -1
    assert bwd(act=9) == -10 and bwd(w=MIS16) == -7 and bwd(vdz=vh) == -2 and bwd(vh=vx, h=P4) == -2 and bwd(vz=view(C=12, W=5)) == -2
    assert bwd(vdz=dc.View.q8(2, 24, 4, 6)) == -3 and bwd(vz=q, zu=MIS16) == -7
    deep = view(C=(1 << 19) + 1)
    assert bwd(vz=deep) == -11


def test_join_refusals():
    v, w, q = view(), view(C=9), dc.View.q8(2, 8, 4, 6)
    n = dc.Norm(dc.DC_NORM_LAYER, 1e-5)
    base = dict(vy=v, y=P1, post=n, scale=None, gate=None, drop=None, vx=v, x=P2, pre=n, vo=v, o=P3, vu=v, u=P4, stat=None, ckpt=None,
                stream=0)
    fwd = with_(dc.join_fwd, base)
    for k in ("vy", "y", "vx", "vo", "o", "vu", "u"):
        assert fwd(**{k: None}) == -1, k
    assert fwd(vx=w) == -2 and fwd(vo=w) == -2 and fwd(vu=w) == -2 and fwd(vy=q) == -3 and fwd(vo=q) == -3
    assert fwd(pre=None) == -10                                   # u without a norm
    assert fwd(vo=view(sc=23)) == -2 and fwd(vu=view(sn=0)) == -2
    for bad in (dc.Norm(3, 1e-5), dc.Norm(-1, 1e-5), dc.Norm(1, -1.0), dc.Norm(2, float("nan")), dc.Norm(1, float("inf"))):
        assert fwd(post=bad) == -10 and fwd(pre=bad) == -10
    assert fwd(post=dc.Norm(1, 1e-5, MIS16)) == -7 and fwd(pre=dc.Norm(2, 1e-5, None, MIS16)) == -7
    for k in ("scale", "gate", "stat", "ckpt"):
        assert fwd(**{k: MIS16}) == -7, k
    assert fwd(y=MIS2) == -7 and fwd(u=MIS2) == -7
    need = dc.join_bwd_workspace_bytes(v, True)
    assert need > 0 and need % 16 == 0 and dc.join_bwd_workspace_bytes(view(N=0), True) == 0
    G = dc.JoinGrads
    base = dict(vdu=v, du=P1, vdo=v, do=P1, vy=v, y=P2, vx=v, x=P2, vo=None, o=None, stat=P4, post=n, scale=None, gate=P4, drop=None, pre=n, vdx=v, dx=P3,
                vdy=v, dy=P4, grads=G(scale=P1), accumulate=0, workspace=Ws(need), stream=0)
    bwd = with_(dc.join_bwd, base)
    for k in ("vdu", "vdo", "vy", "y", "vx", "stat", "vdx", "vdy", "dy"):
        assert bwd(**{k: None}) == -1, k
    assert bwd(o=P3) == -1 and bwd(post=None, y=None, grads=None) == -1      # o is formed from y
    assert bwd(du=None, do=None) == -1
    assert bwd(du=None, pre=None, post=None, y=None) == -1        # a gradient of scale reads y
    assert bwd(pre=None) == -10 and bwd(post=dc.Norm(5, 0.0)) == -10 and bwd(accumulate=2) == -10
    for k in ("vdu", "vdo", "vy", "vx", "vdx"):
        assert bwd(**{k: w}) == -2, k
    assert bwd(vo=w, o=P3) == -2 and bwd(vx=q, x=MIS16) == -7
    assert bwd(vdu=q) == -3 and bwd(vdx=q) == -3 and bwd(vdy=q) == -3 and bwd(vy=q, y=MIS16) == -7 and bwd(vo=q, o=MIS16) == -7
    # gradients of parameters that the call has not
    assert bwd(gate=None, grads=G(gate=P1)) == -10 and bwd(post=None, grads=G(gamma_post=P1)) == -10
    assert bwd(du=None, grads=G(gamma_pre=P1)) == -10 and bwd(du=None, grads=G(beta_pre=P1)) == -10
    for k in ("scale", "gate", "gamma_post", "beta_post", "gamma_pre", "beta_pre"):
        assert bwd(grads=G(**{k: MIS16})) == -7, k
    assert bwd(workspace=None) == -6 and bwd(workspace=Ws(need - 1)) == -6 and bwd(workspace=Ws(need, MIS16)) == -7
    assert bwd(stat=MIS16) == -7 and bwd(gate=MIS16) == -7


def test_python_structs_are_the_header_s():
    assert ctypes.sizeof(dc.Drop) == 64 and (dc.Drop.seed.offset, dc.Drop.step.offset, dc.Drop.n0.offset, dc.Drop.Q.offset) == (8, 24, 32, 56)
    assert ctypes.sizeof(dc.Norm) == 24 and dc.Norm.eps.offset == 4
    assert ctypes.sizeof(dc.JoinGrads) == 48
    t = torch.zeros(4)
    assert dc.JoinGrads(gamma_pre=t)._gamma_pre == t.data_ptr() and dc.Norm(1, 0.5, None, t)._beta == t.data_ptr()


# ------------------------------------------------------------------ the oracles themselves

# the generator's known answers, as its authors publish them
VECTORS = [([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
           ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
           ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])]


@pytest.mark.parametrize("ctr,key,want", VECTORS)
def test_generator_of_the_oracle(ctr, key, want):
    assert R.philox(ctr, key) == want
    pos, off, seed = ctr[0] | ctr[1] << 32, ctr[2] | ctr[3] << 32, key[0] | key[1] << 32
    assert R._philox_array(np.array([pos], dtype=np.uint64), off, seed)[0].tolist() == want


def test_mask_of_the_oracle():
    """Shares, factors, and a tile's mask as a part of the whole one's."""
    m = R.mask((2, 20, 12, 16), 0.3, 7, 5)
    t = round(65536 * 0.3)
    assert set(m.unique().tolist()) == {0.0, 65536 / (65536 - t)}
    assert abs(float((m == 0).double().mean()) - t / 65536) < 4 * (0.3 * 0.7 / m.numel()) ** 0.5     # four deviations
    whole = m.view(2, 20, 12, 16)
    for h0, w0, h, w in ((0, 0, 12, 16), (3, 5, 4, 7), (11, 15, 1, 1)):
        part = R.mask((1, 20, h, w), 0.3, 7, 5, n0=1, h0=h0, w0=w0, H=12, W=16).view(1, 20, h, w)
        assert torch.equal(part, whole[1:, :, h0:h0 + h, w0:w0 + w])
    tiles = R.mask((4, 20, 6, 8), 0.3, 7, 5, P=2, Q=1, W=16).view(2, 2, 20, 6, 8)        # left half, two rows of tiles
    assert torch.equal(tiles[1, 1], whole[1, :, 6:, :8])
    assert not torch.equal(R.mask((2, 20, 12, 16), 0.3, 7, 6), m)
    assert torch.equal(R.mask((2, 20, 12, 16), 0.3, 7, 3, step=2), m)


def test_gate_gradients_against_automatic_ones():
    g = torch.Generator().manual_seed(1)

    def randn(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    for kind in ("none", "relu", "gelu", "silu"):
        x, w, b, w2, dy = randn(2, 5, 6), randn(8, 5), randn(8), randn(3, 4), randn(2, 3, 6)
        m = (torch.rand(2, 4, 6, generator=g) > 0.3) * 1.5
        z = torch.einsum("kc,ncp->nkp", w, x) + b[:, None]
        z.requires_grad_()
        h = R.act(z[:, :4], kind) * z[:, 4:] * m
        (torch.einsum("kc,ncp->nkp", w2, h) * dy).sum().backward()
        zg, zu, _, _ = R.gate_sums(x, w, b)
        dg, du, h2, *_ = R.gate_bwd(dy, w2, zg, zu, kind, m)
        assert torch.allclose(torch.cat((dg, du), 1), z.grad, rtol=1e-10, atol=1e-12) and torch.allclose(h2, h.detach(), rtol=1e-12)
        assert torch.allclose(R.gate(zg, zu, 0 * zg, 0 * zu, kind, m)[0], h2, rtol=1e-12)


def _join_inputs(seed):
    g = torch.Generator().manual_seed(seed)

    def randn(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    a = {"y": randn(2, 7, 5), "x": randn(2, 7, 5), "scale": randn(7), "gate": randn(2, 7), "gamma_post": randn(7), "beta_post": randn(7),
         "gamma_pre": randn(7), "beta_pre": randn(7)}
    return a, (torch.rand(2, 7, 5, generator=g) > 0.3) * 1.5, randn(2, 7, 5), randn(2, 7, 5)


@pytest.mark.parametrize("post,pre", [("layer", "rms"), ("rms", "layer"), (None, "layer"), ("rms", None), (None, None)])
def test_join_gradients_against_automatic_ones_and_differences(post, pre):
    a, m, du, do = _join_inputs(3)

    def norms(a):
        return [(k, a["gamma_" + s], a["beta_" + s]) if k else None for k, s in ((post, "post"), (pre, "pre"))]

    def loss(a):
        n = norms(a)
        out = R.join(a["y"], n[0], (a["scale"] * a["gate"])[:, :, None], m, a["x"], n[1], 1e-5)
        return (out["o"][0] * do).sum() + ((out["u"][0] * du).sum() if pre else 0), out["o"][0]

    leaf = {k: t.clone().requires_grad_() for k, t in a.items()}
    total, o = loss(leaf)
    total.backward()
    stat = [R.moments(t, k, 1e-5) if k else None for t, k in ((a["y"], post), (o.detach(), pre))]
    n = norms(a)
    got = R.join_bwd(du if pre else None, do, a["y"], o.detach(), stat, n[0], a["scale"], a["gate"], m, n[1])
    pairs = [("dx", "x"), ("dy", "y"), ("scale", "scale"), ("gate", "gate")] + [(f"{k}_{s}", f"{k}_{s}") for s, on in
                                                                             (("post", post), ("pre", pre)) if on for k in ("gamma", "beta")]
    g = torch.Generator().manual_seed(4)
    for name, key in pairs:
        assert torch.allclose(got[name][0], leaf[key].grad, rtol=1e-9, atol=1e-10), name
        d = torch.randn(a[key].shape, generator=g, dtype=torch.float64)
        num = (loss({**a, key: a[key] + 1e-5 * d})[0] - loss({**a, key: a[key] - 1e-5 * d})[0]) / 2e-5
        assert abs(float((got[name][0] * d).sum() - num)) < 1e-6 * max(1, abs(float(num))), name


def test_norms_of_the_oracle():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(2, 9, 4, generator=g, dtype=torch.float64)
    ga, be = torch.randn(9, generator=g, dtype=torch.float64), torch.randn(9, generator=g, dtype=torch.float64)
    want = A.norm(x.numpy(), ga.numpy(), be.numpy(), 1e-5)[0]
    assert np.allclose(R.norm(x, "layer", ga, be, 1e-5)[0].numpy(), want, rtol=1e-12)
    u, mu, r = R.norm(x, "rms", ga, be, 0.0)
    assert not mu.any() and np.allclose((((u - be[:, None]) / ga[:, None]) ** 2).mean(1).numpy(), 1.0)
