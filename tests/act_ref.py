"""Plain 64-bit forms of the operators between two convolutions, the byte layout of
the 8-bit checkpoint, and tensors in the layouts that the library takes.  Shares no
code with the library."""
import math

import numpy as np
import torch

EPS32 = 2.0 ** -24      # rounding of an fp32 operation, relative
BF = 2.0 ** -8          # of a result to bf16 (8 significant bits)


def q8_values(x):
    """What x [N][C][pixels] (float64, numpy) stands for in 8 bits."""
    N, C, P = x.shape
    cb = -(-C // 32)
    b = np.zeros((N, cb * 32, P))
    b[:, :C] = x
    b = b.reshape(N, cb, 32, P)
    with np.errstate(invalid="ignore"):
        top = np.abs(b).max(2, keepdims=True)
    bad = ~np.isfinite(top)
    power = np.where((top > 0) & ~bad, np.frexp(np.where(bad, 1.0, top))[1] - 1, -1000)
    power = np.maximum(power, -120)
    step = np.ldexp(1.0, power - 6)
    with np.errstate(invalid="ignore"):
        v = np.clip(np.rint(b / step), -127, 127) * step      # rint: ties to even
    v = np.where(bad, np.nan, v)
    return v.reshape(N, cb * 32, P)[:, :C]


def q8_decode(buf, N, C, P):
    """The values that the bytes of a checkpoint stand for, by the documented layout."""
    cb = -(-C // 32)
    raw = buf.cpu().numpy().view(np.uint8)
    q = raw[:N * cb * P * 32].view(np.int8).reshape(N, cb, P, 32).astype(np.float64)
    s = raw[N * cb * P * 32:N * cb * P * 33].reshape(N, cb, P).astype(np.int64)
    assert s.min() >= 7
    v = np.where((s == 255)[..., None], np.nan, q * np.ldexp(1.0, s - 133)[..., None])
    if C % 32:
        assert not q[:, -1, :, C % 32:].any()
    return v.transpose(0, 1, 3, 2).reshape(N, cb * 32, P)[:, :C]


_erf = np.vectorize(math.erf)


def act(z, kind):
    if kind == "relu":
        return np.where(z > 0, z, 0 * z)
    if kind == "gelu":
        return z * 0.5 * (1 + _erf(z / math.sqrt(2)))
    if kind == "silu":
        return z / (1 + np.exp(-z))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        e = np.exp(-z)
        return (1 + e + z * e) / (1 + e) ** 2
    return np.ones_like(z)


def norm(x, gamma, beta, eps):
    """x [N][C][pixels] -> u, mu, r."""
    mu = x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)
    return gamma[:, None] * (x - mu) * r + beta[:, None], mu, r


def norm_bwd(du, x, mu, r, gamma):
    xh = (x - mu) * r
    g = gamma[:, None] * du
    dx = r * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (du * xh).sum((0, 2)), du.sum((0, 2)), xh


DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def tensor(layout, N, C, H, W, dtype, device="cuda", fill=float("nan")):
    """An [N][C][H][W] view of memory full of `fill`, and the memory."""
    dt = DT[dtype]

    def full(*shape):
        return torch.full(shape, fill, dtype=dt, device=device)

    if layout == "dense":
        t = full(N, C, H, W)
        return t, t
    if layout == "padded":      # the interior of a tile with a margin of 1 and 16-byte rows
        per = 16 // dt.itemsize
        t = full(N, C, H + 2, -(-(W + 2) // per) * per)
        return t[:, :, 1:1 + H, 1:1 + W], t
    if layout == "gaps":        # rows, channels and samples with odd gaps, from an odd start
        t = full(N * 2 * (C + 3) * (H + 1) * (W + 3) + 5)
        v = torch.as_strided(t, (N, C, H, W), (2 * (C + 3) * (H + 1) * (W + 3), (H + 1) * (W + 3), W + 3, 1), 5)
        return v, t
    if layout == "rows":        # channels contiguous: rows of channels
        assert W == 1
        t = full(N, H, C)
        return t.permute(0, 2, 1).unsqueeze(3), t
    if layout == "slice":       # rows of channels inside wider ones
        assert W == 1
        t = full(N, H, C + 8)
        return t[:, :, 8:].permute(0, 2, 1).unsqueeze(3), t
    raise ValueError(layout)


def f64(t):
    """[N][C][H][W] tensor -> [N][C][pixels] float64."""
    return t.detach().float().cpu().numpy().astype(np.float64).reshape(t.shape[0], t.shape[1], -1)


def untouched(view, memory, fill_is_nan=True):
    """Whether the memory outside the view still holds its fill (NaN)."""
    m = memory.clone()
    v = torch.as_strided(m, view.shape, view.stride(), view.storage_offset() - memory.storage_offset())
    v.fill_(float("nan"))
    return bool(torch.isnan(m).all())


def close(got, ref, tol, what):
    """|got - ref| <= tol where ref is finite; the same NaN and infinities elsewhere."""
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), what
    err, bound = np.abs(got - ref)[fine], np.broadcast_to(tol, ref.shape)[fine]
    if err.size:
        k = np.argmax(err - bound)
        assert (err <= bound).all(), f"{what}: {err[k]:.3e} off where {bound[k]:.3e} is allowed"
