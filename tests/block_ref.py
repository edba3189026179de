"""Plain 64-bit forms of a gated residual block's operators (torch, any device) on tensors
[N][C][pixels], with bounds for what fp32 sums may be off.  Shares no code with the library."""
import math

import numpy as np
import torch

EPS32 = 2.0 ** -24      # rounding of an fp32 operation, relative
BF = 2.0 ** -8          # of a result to bf16


# ------------------------------------------------------------------ dropout

def philox(ctr, key):
    """Philox 4x32 with 10 rounds, on Python integers: four words and two."""
    c, k = list(ctr), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def _philox_array(pos, ctr, seed):
    """The same for an array of positions (uint64), [...][4] words."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [pos & low, pos >> half, np.full_like(pos, ctr & 0xFFFFFFFF), np.full_like(pos, ctr >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def threshold(p):
    return min(int(np.rint(65536 * np.float64(p))), 65535)


def mask(shape, p, seed, offset=0, step=0, n0=0, h0=0, w0=0, H=0, W=0, P=0, Q=0, device="cpu"):
    """What a tensor [N][C][h][w] is multiplied by, [N][C][pixels]."""
    N, C, h, w = shape
    P, Q = max(P, 1), max(Q, 1)
    H, W = H or h0 + P * h, W or w0 + Q * w
    t, G, per = threshold(p), -(-C // 8), N // (P * Q)
    i = np.arange(N)
    tile, n = i // per, n0 + i % per
    row = h0 + (tile // Q)[:, None] * h + np.arange(h)            # [N][h]
    col = w0 + (tile % Q)[:, None] * w + np.arange(w)             # [N][w]
    pos = ((n[:, None, None, None] * G + np.arange(G)[:, None, None]) * H + row[:, None, :, None]) * W + col[:, None, None, :]
    words = _philox_array(pos.astype(np.uint64), (offset + step) % 2 ** 64, seed)    # [N][G][h][w][4]
    sixteen = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(N, G, h * w, 8)
    keep = (sixteen >= t).transpose(0, 1, 3, 2).reshape(N, G * 8, h * w)[:, :C]
    return torch.from_numpy(keep * (65536 / (65536 - t))).to(device)


# ------------------------------------------------------------------ the gated product

def act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, 0 * z)
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    return z * torch.sigmoid(z) if kind == "silu" else z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def product(w, x):
    """w [K][C] times x [N][C][pixels]."""
    return (w @ x.transpose(0, 1).flatten(1)).view(w.shape[0], x.shape[0], -1).transpose(0, 1)


def gate_sums(x, w, b):
    """zg, zu and their errors: C products and the bias, in fp32."""
    z, top = product(w, x) + b[:, None], product(w.abs(), x.abs()) + b.abs()[:, None]
    K = w.shape[0] // 2
    e = (x.shape[1] + 2) * EPS32 * top
    return z[:, :K], z[:, K:], e[:, :K], e[:, K:]


def gate(zg, zu, eg, eu, kind, m):
    """h and its bound.  Slopes are at most 1.13, an activation's own error at most 4e-7 |z|; the
    product and the factor round once each."""
    a = act(zg, kind)
    ea = 1.13 * eg + 4e-7 * zg.abs()
    h = a * zu * m
    return h, m * (zu.abs() * ea + a.abs() * eu + ea * eu) + 4 * EPS32 * h.abs()


def gate_bwd(dy, w2, zg, zu, kind, m):
    """dzg, dzu, h from what was kept, and bounds: the product's sum, 1e-6 for the slope's own error."""
    p = product(w2.t().contiguous(), dy)
    ep = (dy.shape[1] + 2) * EPS32 * product(w2.abs().t().contiguous(), dy.abs())
    a, s = act(zg, kind), slope(zg, kind)
    dg, du, h = p * m * zu * s, p * m * a, a * zu * m
    eg = m * zu.abs() * (1.13 * ep + 1e-6 * p.abs()) + 6 * EPS32 * dg.abs()
    eu = m * (a.abs() * ep + 4e-7 * (zg * p).abs()) + 6 * EPS32 * du.abs()
    return dg, du, h, eg, eu, m * 4e-7 * (zg * zu).abs() + 4 * EPS32 * h.abs()


# ------------------------------------------------------------------ norms and the join

def moments(x, kind, eps):
    mu = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    return mu, 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)


def norm(x, kind, gamma, beta, eps):
    mu, r = moments(x, kind, eps)
    return gamma[:, None] * (x - mu) * r + beta[:, None], mu, r


def norm_tol(x, mu, r, gamma, beta):
    """The mean and the centred values are within (C + 8) 2^-24 of the pixel's largest value, times r
    gamma; the variance's own error is relative and smaller still."""
    C = x.shape[1]
    top, xh = x.abs().amax(1, keepdim=True), ((x - mu) * r).abs()
    return EPS32 * gamma.abs()[:, None] * ((C + 8) * top * r * (1 + xh * xh.mean(1, keepdim=True)) + (C + 16) * xh) \
        + 2 * EPS32 * beta.abs()[:, None]


def norm_carried(e, x, mu, r, gamma, kind):
    """What an error e of its input adds to a norm's result, to first order."""
    xh = ((x - mu) * r).abs()
    e = e + (e.mean(1, keepdim=True) if kind == "layer" else 0)
    return 1.01 * gamma.abs()[:, None] * r * (e + xh * (xh * e).mean(1, keepdim=True))


def norm_bwd(g, x, mu, r, gamma, kind):
    """Gradient at x and the normed x, from statistics that are handed over."""
    xh, g = (x - mu) * r, gamma[:, None] * g
    m1 = g.mean(1, keepdim=True) if kind == "layer" else 0
    return r * (g - m1 - xh * (g * xh).mean(1, keepdim=True)), xh


def norm_bwd_tol(g, x, mu, r, gamma, kind, e=0.0):
    """Bounds for both: the normed x takes two roundings of its operands (and x's own error e), the means
    sums of C products."""
    C = x.shape[1]
    xh = ((x - mu) * r).abs()
    ex = 3 * EPS32 * r * (x.abs() + mu.abs()) + r * e
    gd = (gamma[:, None] * g).abs()
    m1 = gd.mean(1, keepdim=True) if kind == "layer" else 0
    m2 = (gd * xh).mean(1, keepdim=True)
    em2 = (C + 8) * EPS32 * m2 + (gd * ex).mean(1, keepdim=True)
    return r * (8 * EPS32 * gd + (C + 8) * EPS32 * m1 + xh * em2 + (ex + 4 * EPS32 * xh) * m2), ex


def norm_bwd_carried(e, x, mu, r, gamma, kind):
    """What an error e of the gradient adds."""
    xh, e = ((x - mu) * r).abs(), gamma.abs()[:, None] * e
    m1 = e.mean(1, keepdim=True) if kind == "layer" else 0
    return 1.01 * r * (e + m1 + xh * (e * xh).mean(1, keepdim=True))


def join(y, post, f, m, x, pre, eps):
    """o and u, with post and pre (kind, gamma, beta) or None, f = scale gate, m the mask.  Returns
    {name: (value, bound)} for o, u and the statistics."""
    out = {}
    v, ev = y, torch.zeros_like(y)
    if post:
        v, mu, r = norm(y, *post, eps)
        ev = norm_tol(y, mu, r, post[1], post[2])
        out["stat"] = stat_bounds(y, mu, r, torch.zeros_like(y))
    b = f * m * v
    o = x + b
    eo = (f * m).abs() * ev + 6 * EPS32 * b.abs() + 2 * EPS32 * o.abs()
    out["o"] = (o, eo)
    if pre:
        u, mu, r = norm(o, *pre, eps)
        out["u"] = (u, norm_tol(o, mu, r, pre[1], pre[2]) + norm_carried(eo, o, mu, r, pre[1], pre[0]))
        out["stat2"] = stat_bounds(o, mu, r, eo)
    return out


def stat_bounds(x, mu, r, e):
    C = x.shape[1]
    top, xh = x.abs().amax(1, keepdim=True), ((x - mu) * r).abs()
    emu = (C + 2) * EPS32 * top + e.mean(1, keepdim=True)
    er = r * (EPS32 * (8 + C + (C + 8) * top * r * 2) + 1.01 * r * (xh * (e + e.mean(1, keepdim=True))).mean(1, keepdim=True))
    return (mu, emu), (r, er)


def join_bwd(du, dr, y, o, stat, post, scale, gate, m, pre, eo=0.0):
    """{name: (value, bound)} of the gradients; stat: (mu, r) of y and of o as the forward pass wrote
    them.  scale [C], gate [N][C]; du and dr may be None; eo: what o may be off."""
    out = {}
    M = m.shape[0] * m.shape[2]
    N = m.shape[0]
    f = (scale * gate)[:, :, None] * m
    d, ed = (dr, torch.zeros_like(dr)) if dr is not None else (0.0, 0.0)
    if du is not None:
        g, xh = norm_bwd(du, o, *stat[1], pre[1], pre[0])
        eg, ex = norm_bwd_tol(du, o, *stat[1], pre[1], pre[0], eo)
        d, ed = d + g, eg
        out["gamma_pre"] = ((du * xh).sum((0, 2)), (M + 4) * EPS32 * (du * xh).abs().sum((0, 2)) + (du.abs() * ex).sum((0, 2)))
        out["beta_pre"] = (du.sum((0, 2)), (M + 4) * EPS32 * du.abs().sum((0, 2)))
    ed = ed + 2 * EPS32 * d.abs()
    out["dx"] = (d, ed)
    dv, edv = d * f, f.abs() * ed + 4 * EPS32 * (d * f).abs()
    v, ev = y, torch.zeros_like(y)
    if post:
        g, xh = norm_bwd(dv, y, *stat[0], post[1], post[0])
        eg, ex = norm_bwd_tol(dv, y, *stat[0], post[1], post[0])
        out["dy"] = (g, eg + norm_bwd_carried(edv, y, *stat[0], post[1], post[0]) + 2 * EPS32 * g.abs())
        out["gamma_post"] = ((dv * xh).sum((0, 2)), (M + 4) * EPS32 * (dv * xh).abs().sum((0, 2)) +
                             (dv.abs() * ex + edv * xh.abs()).sum((0, 2)))
        out["beta_post"] = (dv.sum((0, 2)), (M + 4) * EPS32 * dv.abs().sum((0, 2)) + edv.sum((0, 2)))
        v = post[1][:, None] * xh + post[2][:, None]
        ev = post[1].abs()[:, None] * ex + 4 * EPS32 * (v.abs() + post[2].abs()[:, None])
    else:
        out["dy"] = (dv, edv)
    t, et = d * v * m, m * (ed * v.abs() + d.abs() * ev) + 4 * EPS32 * (d * v * m).abs()
    size, err = t.abs().sum(2), et.sum(2)
    out["gate"] = (scale * t.sum(2), scale.abs() * ((m.shape[2] + 6) * EPS32 * size + err))
    out["scale"] = ((gate * t.sum(2)).sum(0), (gate.abs() * ((M + N + 6) * EPS32 * size + err)).sum(0))
    return out
