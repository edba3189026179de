"""Host-side checks of the operators between two convolutions: refusals before any
launch, sizes, and the gradients' formulas (the oracles of the GPU tests) against
differences.  No GPU."""
import ctypes

import numpy as np
import pytest
import torch

import act_ref as R
import paper_1903_06681_amd as dc

A, B, D, MIS2, MIS16 = 0x10000, 0x20000, 0x30000, 0x10001, 0x10008


def view(N=2, C=8, H=4, W=6, sn=None, sc=None, sh=None, dtype=dc.DC_F32):
    sh = W if sh is None else sh
    sc = H * sh if sc is None else sc
    return dc.View(N, C, H, W, C * sc if sn is None else sn, sc, sh, dtype)


def status(fn, *args):
    with pytest.raises(dc.DcError) as e:
        fn(*args)
    return e.value.status


class Ws:
    def __init__(self, n, ptr=A):
        self.n, self.ptr = n, ptr

    def numel(self):
        return self.n

    def element_size(self):
        return 1

    def data_ptr(self):
        return self.ptr


def test_view_of_tensors():
    t = torch.empty(2, 3, 5, 7)
    v = dc.View.of(t)
    assert (v.N, v.C, v.H, v.W, v.sn, v.sc, v.sh, v.dtype) == (2, 3, 5, 7, 105, 35, 7, dc.DC_F32)
    v = dc.View.of(t.bfloat16()[:, 1:, 1:4, 2:])
    assert (v.C, v.H, v.W, v.sc, v.sh, v.dtype) == (2, 3, 5, 35, 7, dc.DC_BF16)
    for bad in (t[0], t.half(), t[:, :, :, ::2], t.transpose(2, 3)):
        with pytest.raises(ValueError):
            dc.View.of(bad)


def test_ckpt_bytes():
    for N, C, P in ((1, 1, 1), (2, 32, 5), (3, 33, 77)):
        want = -(-N * -(-C // 32) * P * 33 // 16) * 16
        assert dc.ckpt_bytes(dc.View.q8(N, C, 1, P)) == want
    assert dc.ckpt_bytes(dc.View.q8(0, 1, 1, 1)) == -1


@pytest.mark.parametrize("kw,code", [
    ({"N": 0}, -2), ({"C": -1}, -2), ({"H": 0}, -2), ({"W": 0}, -2), ({"dtype": 3}, -3), ({"dtype": dc.DC_Q8}, -3),
    ({"sc": -24}, -2), ({"sh": -6}, -2), ({"N": 1 << 16, "H": 1 << 8, "W": 1 << 8}, -11), ({"C": (1 << 20) + 1}, -11),
    ({"N": 3, "sn": 1 << 62}, -11),
])
def test_bad_views(kw, code):
    v, good = view(**kw), view()
    assert status(dc.ckpt_save, v, A, B, 0) == code
    assert status(dc.norm_fwd, v, A, None, None, 1e-5, v if code != -2 or kw.get("N") == 0 else good, B, None, None, 0) == code
    assert status(dc.linear_fwd, v, A, B, None, 0, None, None, None, None, good, D, 0) == code


@pytest.mark.parametrize("kw", [{"sh": 5}, {"sc": 23}, {"sn": 0}, {"sh": 0}, {"sn": 30, "sc": 24, "sh": 6}])
def test_written_views_must_not_overlap(kw):
    v, good = view(**kw), view()
    assert status(dc.norm_fwd, good, A, None, None, 1e-5, v, B, None, None, 0) == -2
    assert status(dc.linear_fwd, good, A, B, None, 0, None, None, None, None, v, D, 0) == -2
    assert status(dc.ckpt_load, dc.View.q8(2, 8, 4, 6), A, 0, v, B, 0) == -2
    assert status(dc.linear_bwd_data, good, A, B, 0, None, None, None, None, v, D, 0) == -2


def test_ckpt_refusals():
    v, q = view(), dc.View.q8(2, 8, 4, 6)
    assert status(dc.ckpt_save, None, A, B, 0) == -1
    assert status(dc.ckpt_save, v, None, B, 0) == -1
    assert status(dc.ckpt_save, v, A, None, 0) == -1
    assert status(dc.ckpt_save, v, A, MIS16, 0) == -7
    assert status(dc.ckpt_save, v, MIS2, B, 0) == -7
    assert status(dc.ckpt_load, v, A, 0, v, B, 0) == -3
    assert status(dc.ckpt_load, q, A, 4, v, B, 0) == -10
    assert status(dc.ckpt_load, q, A, 0, view(C=9), B, 0) == -2
    assert status(dc.ckpt_load, q, A, 0, None, B, 0) == -1
    assert status(dc.ckpt_load, q, None, 0, v, B, 0) == -1


def test_norm_refusals():
    v, w = view(), view(C=9)
    ok = (v, A, None, None, 1e-5, v, B, None, None, 0)

    def fwd(**kw):
        names = ("vx", "x", "gamma", "beta", "eps", "vu", "u", "stat", "ckpt", "stream")
        return status(dc.norm_fwd, *(kw.get(n, o) for n, o in zip(names, ok)))

    assert fwd(vx=None) == -1 and fwd(x=None) == -1 and fwd(u=None) == -1 and fwd(vu=None) == -1
    assert fwd(vu=w) == -2 and fwd(eps=-1.0) == -10 and fwd(eps=float("nan")) == -10 and fwd(eps=float("inf")) == -10
    assert fwd(gamma=MIS16) == -7 and fwd(beta=MIS16) == -7 and fwd(stat=MIS16) == -7 and fwd(ckpt=MIS16) == -7
    assert fwd(u=MIS2) == -7
    need = dc.norm_bwd_workspace_bytes(v)
    assert need > 0 and need % 16 == 0
    base = dict(vdu=v, du=A, vx=v, x=A, stat=A, gamma=None, beta=None, vres=None, res=None, vu=None, u=None, vdx=v, dx=B,
                dgamma=A, dbeta=A, accumulate=0, workspace=Ws(need), stream=0)

    def bwd(**kw):
        return status(dc.norm_bwd, *{**base, **kw}.values())

    assert bwd(du=None) == -1 and bwd(vdu=None) == -1 and bwd(x=None) == -1 and bwd(stat=None) == -1 and bwd(dx=None) == -1
    assert bwd(vx=w) == -2 and bwd(vdx=w) == -2 and bwd(vres=w, res=A) == -2 and bwd(vu=w, u=A) == -2
    assert bwd(vres=None, res=A) == -1
    assert bwd(accumulate=2) == -10
    assert bwd(workspace=None) == -6 and bwd(workspace=Ws(need - 1)) == -6 and bwd(workspace=Ws(need, MIS16)) == -7
    assert bwd(dgamma=MIS16) == -7 and bwd(stat=MIS16) == -7
    assert bwd(vdu=dc.View.q8(2, 8, 4, 6)) == -3 and bwd(vdx=dc.View.q8(2, 8, 4, 6)) == -3
    assert bwd(vx=dc.View.q8(2, 8, 4, 6), x=MIS16) == -7
    assert dc.norm_bwd_workspace_bytes(view(N=0)) == 0


def test_linear_refusals():
    vx, vy = view(), view(C=12)
    base = dict(vx=vx, x=A, w=B, bias=None, act=0, vres=None, res=None, vz=None, z=None, vy=vy, y=D, stream=0)

    def fwd(**kw):
        return status(dc.linear_fwd, *{**base, **kw}.values())

    assert fwd(vx=None) == -1 and fwd(x=None) == -1 and fwd(w=None) == -1 and fwd(y=None) == -1 and fwd(vy=None) == -1
    assert fwd(act=-1) == -10 and fwd(act=4) == -10
    assert fwd(w=MIS16) == -7 and fwd(bias=MIS16) == -7
    assert fwd(vy=view(C=12, H=3)) == -2 and fwd(vres=vx, res=A) == -2 and fwd(vz=vx, z=A) == -2 and fwd(z=A) == -1
    assert fwd(vy=dc.View.q8(2, 12, 4, 6)) == -3 and fwd(vres=dc.View.q8(2, 12, 4, 6), res=A) == -3
    assert fwd(vz=dc.View.q8(2, 12, 4, 6), z=MIS16) == -7
    base = dict(vdy=vy, dy=A, w=B, act=2, vz=vx, z=A, vh=None, h=None, vdx=vx, dx=D, stream=0)

    def bwd(**kw):
        return status(dc.linear_bwd_data, *{**base, **kw}.values())

    assert bwd(dy=None) == -1 and bwd(w=None) == -1 and bwd(dx=None) == -1 and bwd(z=None) == -1 and bwd(vz=None) == -1
    assert bwd(act=0) == -10 and bwd(act=0, vz=None, z=None, vh=vx, h=A) == -10 and bwd(act=9) == -10
    assert bwd(vz=vy) == -2 and bwd(vh=vy, h=A) == -2 and bwd(vdx=view(W=5)) == -2
    assert bwd(w=MIS16) == -7
    need = dc.linear_bwd_filter_workspace_bytes(view(H=64, W=64), view(C=12, H=64, W=64))
    assert need > 0
    base = dict(vx=view(H=64, W=64), x=A, vdy=view(C=12, H=64, W=64), dy=A, dw=B, db=D, accumulate=0, workspace=Ws(need), stream=0)

    def wg(**kw):
        return status(dc.linear_bwd_filter, *{**base, **kw}.values())

    assert wg(x=None) == -1 and wg(dy=None) == -1 and wg(dw=None) == -1
    assert wg(vx=view()) == -2 and wg(vx=view(H=64, W=64, dtype=dc.DC_BF16)) == -3
    assert wg(accumulate=-1) == -10 and wg(workspace=None) == -6 and wg(workspace=Ws(need - 1)) == -6
    assert wg(workspace=Ws(need, MIS16)) == -7 and wg(dw=MIS16) == -7 and wg(db=MIS16) == -7
    assert dc.linear_bwd_filter_workspace_bytes(view(), view(N=3)) == 0
    # weights of 2^31 elements, and more blocks than a launch takes
    big = view(N=1, H=1, W=1, C=1 << 16)
    assert status(dc.linear_fwd, big, A, B, None, 0, None, None, None, None, big, D, 0) == -11
    long = view(N=1, C=1 << 12, H=1, W=(1 << 31) - (1 << 17), sc=1, sh=0)
    out = view(N=1, C=1, H=1, W=(1 << 31) - (1 << 17))
    assert status(dc.linear_fwd, long, A, B, None, 0, None, None, None, None, out, D, 0) == -11


def test_python_struct_is_the_header_s():
    assert ctypes.sizeof(dc.View) == 48
    assert (dc.View.sn.offset, dc.View.sh.offset, dc.View.dtype.offset) == (16, 32, 40)


# ------------------------------------------------------------------ the oracles themselves

def slope_of(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def test_norm_gradient_against_differences():
    g = np.random.default_rng(1)
    x, gamma, beta, du = g.normal(size=(2, 7, 5)), g.normal(size=7), g.normal(size=7), g.normal(size=(2, 7, 5))
    _, mu, r = R.norm(x, gamma, beta, 1e-5)
    dx, dg, db, _ = R.norm_bwd(du, x, mu, r, gamma)
    for got, at, k in ((dx, x, 0), (dg, gamma, 1), (db, beta, 2)):
        d = g.normal(size=at.shape)
        args = [x, gamma, beta]

        def loss(v):
            return (R.norm(*[v if i == k else a for i, a in enumerate(args)], 1e-5)[0] * du).sum()

        assert abs((got * d).sum() - slope_of(loss, at, d)) < 1e-7 * max(1, abs((got * d).sum()))


@pytest.mark.parametrize("kind", ["relu", "gelu", "silu"])
def test_activation_slopes_against_differences(kind):
    z = np.linspace(-6, 6, 1001) + 1e-3
    assert np.abs(R.slope(z, kind) - slope_of(lambda v: R.act(v, kind), z, 1.0, 1e-6)).max() < 1e-8


def test_product_gradients_against_differences():
    g = np.random.default_rng(2)
    x, w, b, dy = g.normal(size=(2, 5, 6)), g.normal(size=(4, 5)), g.normal(size=4), g.normal(size=(2, 4, 6))

    def loss(x, w, b):
        return (R.act(np.einsum("kc,ncp->nkp", w, x) + b[:, None], "gelu") * dy).sum()

    dz = dy * R.slope(np.einsum("kc,ncp->nkp", w, x) + b[:, None], "gelu")
    grads = np.einsum("kc,nkp->ncp", w, dz), np.einsum("nkp,ncp->kc", dz, x), dz.sum((0, 2))
    for k, got in enumerate(grads):
        d = g.normal(size=got.shape)
        num = slope_of(lambda v: loss(*[v if i == k else a for i, a in enumerate((x, w, b))]), (x, w, b)[k], d)
        assert abs((got * d).sum() - num) < 1e-7 * max(1, abs(num))


def test_8_bit_form_of_the_oracle():
    x = np.zeros((1, 32, 3))
    x[0, :3, 0] = 1.0, -0.9921875, 0.0078125          # 64, -63.5 (a tie: -64), 0.5 (a tie: 0)
    x[0, 0, 1] = 1.9999
    v = R.q8_values(x)
    assert list(v[0, :3, 0]) == [1.0, -1.0, 0.0] and v[0, 0, 1] == 127 / 64 and not v[0, :, 2].any()
