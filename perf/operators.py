"""What a network does between two convolutions, as timed cases: layer norm over a
pixel's channels, the pointwise matrix product with bias, activation and residual in
its epilogue, and activation checkpoints in 8 bits.

A case is one pass of a program that holds a tile (or rows of channels: H = W = 1):

  norm    forward (with the 8-bit checkpoint of the input where `ckpt`), then
          backward with a skip path's gradient: u, dx, dgamma, dbeta, and, from the
          checkpoint, u again (the next product's weight gradient reads it)
  linear  y = act(W x + b) (+ residual)
  train   h = act(z), z = W1 x + b1, z kept in 8 bits (`ckpt`) or whole, then the gradient
          at z from the output's: (W2^T dy) * act'(z), and h again from the kept z
  wgrad   dW = sum over pixels of dy x^T, db = sum over pixels of dy
  ckpt    an activation saved in 8 bits and loaded again

`halo`: the tile that `norm` writes and `linear`, `train` and `wgrad` read is the
interior of one padded for a convolution of that margin; 0 is a dense tile.

The 8-bit form: the 32 channels 32 k .. 32 k + 31 of a pixel share the power of two that
the largest magnitude among them has, at least 2^-120; a value is the nearest multiple
(ties to even) of a 64th of it, at most 127 of them.
"""
import math

import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
#: limits of a drawn case, below those of the largest listed one
MOST_FLOPS = {"bf16": 2.5e11, "f32": 2.5e10}
MOST_BYTES = 5e8


def _case(name, op, dtype, N, C, H, W, K=0, act="none", res=False, ckpt=False, halo=0, xdtype=None):
    c = {"op": op, "dtype": dtype, "N": N, "C": C, "H": H, "W": W, "K": K, "act": act, "res": res, "ckpt": ckpt,
         "halo": halo, "xdtype": xdtype or dtype}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the smallest decomposed layer's tile: latency and launches count
        _case("norm_small_f32", "norm", "f32", 2, 8, 16, 16),
        # after the 3x3 layer of the 256x256 tile: fp32 sums in, the next layer's padded tile out, trained from 8 bits
        _case("norm_tile_bf16", "norm", "bf16", 4, 64, 256, 256, ckpt=True, halo=1, xdtype="f32"),
        # a late stage: many channels on few pixels whose rows end off the alignment
        _case("norm_wide_bf16", "norm", "bf16", 32, 1024, 14, 14, ckpt=True),
        # the classifier on a few pooled samples, as when serving
        _case("linear_head_bf16", "linear", "bf16", 4, 2048, 1, 1, K=1000),
        # a block's product back to the narrow width, the skip path added
        _case("linear_down_res_bf16", "linear", "bf16", 32, 512, 28, 28, K=128, res=True),
        # the mesh model in single precision: a tile's product to the wide width
        _case("linear_mesh_f32", "linear", "f32", 1, 32, 512, 512, K=128, act="gelu"),
        # a first-stage block's wide activation, forward and backward from 8 bits
        _case("train_56_bf16", "train", "bf16", 32, 64, 56, 56, K=256, act="gelu", ckpt=True),
        # the largest: 65536 pixels from 512 channels to 2048, as in a model of rows of channels
        _case("train_large_bf16", "train", "bf16", 16, 512, 64, 64, K=2048, act="gelu", ckpt=True),
        # its weight gradient
        _case("wgrad_large_bf16", "wgrad", "bf16", 16, 512, 64, 64, K=2048),
        # odd image, channel counts that are no powers of two
        _case("wgrad_ragged_bf16", "wgrad", "bf16", 3, 40, 93, 75, K=160),
        # the 256x256 tile's input kept for the backward pass
        _case("ckpt_tile_bf16", "ckpt", "bf16", 4, 64, 256, 256),
        # an odd tile in single precision, the last block of channels not full
        _case("ckpt_ragged_f32", "ckpt", "f32", 3, 40, 93, 75),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    """Mostly whole groups of 8 to 64 channels, now and then any count."""
    c, g = _log(rng, lo, hi), rng.choice((1, 8, 16, 32, 64))
    return max(lo, min(hi, (c + g // 2) // g * g)) if c > g else c


def _draw_one(rng):
    op, dtype = rng.choice(("norm", "linear", "linear", "train", "wgrad", "wgrad", "ckpt")), rng.choice(("f32", "bf16", "bf16"))
    form = rng.choice(("tile", "image", "image", "rows"))
    if form == "tile":       # a decomposed layer's tile
        N, H, W, C, F = rng.randint(1, 4), _log(rng, 16, 512), _log(rng, 16, 512), (8, 128), (8, 256)
    elif form == "image":    # whole images, one GPU's samples
        N, H, W, C, F = _log(rng, 1, 32), _log(rng, 2, 112), _log(rng, 2, 112), (16, 1024), (16, 2048)
    else:                    # one pixel a sample: rows of channels, from a single one on
        N, H, W, C, F = _log(rng, 1, 4096), 1, 1, (64, 2048), (64, 2048)
    halo = rng.choice((0, 0, 1)) if form != "rows" and op != "ckpt" else 0
    # z in 8 bits is for bf16 layers: in fp32 ones a z that two orders of summation round to different
    # eighth bits would make outputs differ by far more than fp32 sums do
    ckpt = rng.random() < 0.6 if op == "norm" else op == "train" and dtype == "bf16" and rng.random() < 0.7
    act = rng.choice(("relu", "gelu", "silu")) if op == "train" else rng.choice(("none", "gelu", "silu")) if op == "linear" else "none"
    return _case(None, op, dtype, N, _channels(rng, *C), H, W, K=_channels(rng, *F) if op in ("linear", "train", "wgrad") else 0,
                 act=act, res=op == "linear" and rng.random() < 0.5, ckpt=ckpt, halo=halo, xdtype=rng.choice(("f32", dtype)) if op == "norm" else dtype)


def draw(rng):
    while True:
        c = _draw_one(rng)
        w = work(c)
        if w["flops"] <= MOST_FLOPS[c["dtype"]] and w["bytes"] <= MOST_BYTES:
            return c


def work(c):
    m, e, ex = c["N"] * c["H"] * c["W"], 4 if c["dtype"] == "f32" else 2, 4 if c["xdtype"] == "f32" else 2
    C, K, q = c["C"], c["K"], 33 / 32
    if c["op"] == "norm":    # x in; u, statistics (and checkpoint) out; du, x (or checkpoint), skip in; dx (and u) out
        fwd = m * C * (ex + e) + 8 * m + 8 * C + (m * C * q if c["ckpt"] else 0)
        bwd = m * C * (3 * e + (q + e if c["ckpt"] else ex)) + 8 * m + 12 * C
        return {"bytes": fwd + bwd, "flops": m * C * 20}
    if c["op"] == "linear":
        return {"bytes": e * (m * C + K * C + m * K * (2 if c["res"] else 1)) + 4 * K, "flops": 2 * m * C * K}
    if c["op"] == "train":   # x, W1 in; h, z out; dy, W2, z in; dz, h out
        return {"bytes": 2 * e * (m * C + K * C) + m * K * (3 * e + 2 * (q if c["ckpt"] else e)) + 4 * K, "flops": 4 * m * C * K}
    if c["op"] == "wgrad":
        return {"bytes": e * m * (C + K) + 4 * K * C + 4 * K, "flops": 2 * m * C * K}
    return {"bytes": m * C * (2 * e + 2 * q), "flops": 4 * m * C}


def _tile(c, channels, dtype, halo):
    """An empty tile: dense, or the interior of one with a margin and 16-byte rows; its margin holds zeros."""
    if not halo:
        return torch.empty(c["N"], channels, c["H"], c["W"], dtype=DTYPES[dtype], device="cuda")
    per = 16 // DTYPES[dtype].itemsize
    pitch = -(-(c["W"] + 2 * halo) // per) * per
    t = torch.zeros(c["N"], channels, c["H"] + 2 * halo, pitch, dtype=DTYPES[dtype], device="cuda")
    return t[:, :, halo:halo + c["H"], halo:halo + c["W"]]


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def filled(channels, dtype, halo=0, offset=0.0):
        t = _tile(c, channels, dtype, halo)
        spread = 0.5 + torch.rand(1, channels, 1, 1, generator=g, device="cuda")   # channels differ in scale and mean
        t.copy_(randn(*t.shape).mul_(spread).add_(offset * randn(1, channels, 1, 1)))
        return t

    C, K, dt = c["C"], c["K"], DTYPES[c["dtype"]]
    s = {"c": c}
    if c["op"] == "norm":
        s["x"] = filled(C, c["xdtype"], offset=0.5)
        s["gamma"], s["beta"] = 1 + 0.2 * randn(C), 0.2 * randn(C)
        s["du"], s["skip"] = filled(C, c["dtype"]), filled(C, c["dtype"])
    elif c["op"] == "linear":
        s["x"] = filled(C, c["dtype"], c["halo"])
        s["w"], s["b"] = (randn(K, C) / math.sqrt(C)).to(dt), 0.2 * randn(K)
        s["skip"] = filled(K, c["dtype"]) if c["res"] else None
    elif c["op"] == "train":
        s["x"], s["dy"] = filled(C, c["dtype"], c["halo"]), filled(C, c["dtype"])
        s["w"], s["b"] = (randn(K, C) / math.sqrt(C)).to(dt), 0.2 * randn(K)
        s["w2"] = (randn(C, K) / math.sqrt(K)).to(dt)
    elif c["op"] == "wgrad":
        s["x"], s["dy"] = filled(C, c["dtype"], c["halo"]), filled(K, c["dtype"])
    else:
        s["x"] = filled(C, c["dtype"], offset=0.5)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program of this library keeps beside its tensors: descriptors of their layout, outputs, checkpoints, workspaces."""
    import paper_1903_06681_amd as dc
    c = s["c"]
    N, C, K, H, W = (c[k] for k in "NCKHW")

    def out(name, channels, halo=0):
        s[name] = _tile(c, channels, c["dtype"], halo)

    def raw(nbytes):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")

    s["act"] = dc.ACT[c["act"]]
    q = s["vq"] = dc.View.q8(N, K if c["op"] == "train" else C, H, W)
    if c["op"] == "norm":
        out("u", C, c["halo"]), out("u2", C), out("dx", C)
        s["stat"] = torch.empty(2, N, H, W, device="cuda")
        s["dgamma"], s["dbeta"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        s["q"] = raw(dc.ckpt_bytes(q)) if c["ckpt"] else None
    elif c["op"] == "linear":
        out("y", K)
    elif c["op"] == "train":
        out("h", K), out("h2", K), out("dz", K)
        if c["ckpt"]:
            s["q"] = raw(dc.ckpt_bytes(q))
        else:
            out("z", K)
    elif c["op"] == "wgrad":
        s["dw"], s["db"] = torch.empty(K, C, device="cuda"), torch.empty(K, device="cuda")
    else:
        out("y", C)
        s["q"] = raw(dc.ckpt_bytes(q))
    for name in ("x", "u", "u2", "du", "dx", "skip", "y", "h", "h2", "z", "dy", "dz"):
        s["v" + name] = dc.View.of(s[name]) if s.get(name) is not None else None
    if c["op"] == "norm":
        s["ws"] = raw(dc.norm_bwd_workspace_bytes(s["vdu"]))
    if c["op"] == "wgrad":
        s["ws"] = raw(dc.linear_bwd_filter_workspace_bytes(s["vx"], s["vdy"]))


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_1903_06681_amd as dc
    c = s["c"]
    if c["op"] == "norm":
        dc.norm_fwd(s["vx"], s["x"], s["gamma"], s["beta"], EPS, s["vu"], s["u"], s["stat"], s["q"])
        vx, x = (s["vq"], s["q"]) if c["ckpt"] else (s["vx"], s["x"])
        vu2, u2 = (s["vu2"], s["u2"]) if c["ckpt"] else (None, None)
        dc.norm_bwd(s["vdu"], s["du"], vx, x, s["stat"], s["gamma"], s["beta"], s["vskip"], s["skip"], vu2, u2,
                    s["vdx"], s["dx"], s["dgamma"], s["dbeta"], 0, s["ws"])
        return {"u": s["u"], "u2": u2, "dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if c["op"] == "linear":
        dc.linear_fwd(s["vx"], s["x"], s["w"], s["b"], s["act"], s["vskip"], s["skip"], None, None, s["vy"], s["y"])
        return s["y"]
    if c["op"] == "train":
        vz, z = (s["vq"], s["q"]) if c["ckpt"] else (s["vz"], s["z"])
        dc.linear_fwd(s["vx"], s["x"], s["w"], s["b"], s["act"], None, None, vz, z, s["vh"], s["h"])
        dc.linear_bwd_data(s["vdy"], s["dy"], s["w2"], s["act"], vz, z, s["vh2"], s["h2"], s["vdz"], s["dz"])
        return {"h": s["h"], "z": s.get("z"), "h2": s["h2"], "dz": s["dz"]}
    if c["op"] == "wgrad":
        dc.linear_bwd_filter(s["vx"], s["x"], s["vdy"], s["dy"], s["dw"], s["db"], 0, s["ws"])
        return {"dw": s["dw"], "db": s["db"]}
    dc.ckpt_save(s["vx"], s["x"], s["q"])
    dc.ckpt_load(s["vq"], s["q"], s["act"], s["vy"], s["y"])
    return s["y"]


# ------------------------------------------------------------- the plain form

def _flat(t):
    return t.float().flatten(2)


def _q8(x):
    """The values that [N][C][pixels] stands for in 8 bits."""
    n, ch, p = x.shape
    b = torch.nn.functional.pad(x, (0, 0, 0, -ch % 32)).view(n, -1, 32, p)
    e = (b.abs().amax(2, keepdim=True).view(torch.int32) >> 23).clamp_(min=7)
    step, per = ((e - 6) << 23).view(torch.float32), ((260 - e) << 23).view(torch.float32)   # powers of two, per = 1 / step
    return ((b * per).round_().clamp_(-127, 127) * step).view(n, -1, p)[:, :ch]


def _product(w, x):
    """w [K][C] times every pixel of x [N][C][pixels]."""
    return torch.matmul(x[:, :, 0], w.t())[:, :, None] if x.shape[2] == 1 else torch.matmul(w, x)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * (0.5 + 0.5 * torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 + 0.5 * torch.erf(z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    sig = torch.sigmoid(z)
    return sig * (1 + z * (1 - sig))


def _run_plain(s):
    c = s["c"]
    dt, shape = DTYPES[c["dtype"]], (c["N"], -1, c["H"], c["W"])

    def tile(t):
        return t.to(dt).view(shape)

    x = _flat(s["x"])
    if c["op"] == "norm":
        g, b = s["gamma"][:, None], s["beta"][:, None]
        d = x - x.mean(1, keepdim=True)
        r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        u, u2 = tile(g * (d * r) + b), None
        xh = (_q8(x) - x.mean(1, keepdim=True)) * r if c["ckpt"] else d * r
        if c["ckpt"]:
            u2 = tile(g * xh + b)
        du = _flat(s["du"])
        gd = g * du
        dx = r * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True)) + _flat(s["skip"])
        return {"u": u, "u2": u2, "dx": tile(dx), "dgamma": (du * xh).sum((0, 2)), "dbeta": du.sum((0, 2))}
    if c["op"] == "linear":
        y = _act(_product(s["w"].float(), x) + s["b"][:, None], c["act"])
        return tile(y + _flat(s["skip"]) if c["res"] else y)
    if c["op"] == "train":
        z = _product(s["w"].float(), x) + s["b"][:, None]
        kept = tile(z)
        zq = _q8(z) if c["ckpt"] else _flat(kept)
        dz = _product(s["w2"].float().t(), _flat(s["dy"])) * _act_slope(zq, c["act"])
        return {"h": tile(_act(z, c["act"])), "z": None if c["ckpt"] else kept, "h2": tile(_act(zq, c["act"])), "dz": tile(dz)}
    if c["op"] == "wgrad":
        dy = _flat(s["dy"]).transpose(0, 1).flatten(1)
        return {"dw": torch.matmul(dy, x.transpose(1, 2).flatten(0, 1)), "db": dy.sum(1)}
    return tile(_q8(x))


# ------------------------------------------------------------- the definition in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    N, H, W = c["N"], c["H"], c["W"]

    def rows(t):                      # pixels by channels
        return t.permute(0, 2, 3, 1).reshape(N * H * W, -1).double()

    def back(r):
        return r.reshape(N, H, W, -1).permute(0, 3, 1, 2)

    def eight_bits(r):
        out = torch.empty_like(r)
        for k in range(0, r.shape[1], 32):
            b = r[:, k:k + 32]
            top = b.abs().max(1, keepdim=True).values
            step = (top / torch.frexp(top).mantissa).nan_to_num(0.0).clamp(min=2.0 ** -119) / 128   # top's own power of two
            out[:, k:k + 32] = torch.clamp(torch.round(b / step), -127, 127) * step
        return out

    def phi(z):
        return torch.special.ndtr(z)

    def act(z):
        return {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0 * z), "gelu": lambda: z * phi(z),
                "silu": lambda: z / (1 + torch.exp(-z))}[c["act"]]()

    def slope(z):
        if c["act"] == "gelu":
            return phi(z) + z * torch.exp(-z * z / 2) * (2 * math.pi) ** -0.5
        if c["act"] == "silu":
            e = torch.exp(-z)
            return (1 + e + z * e) / (1 + e) ** 2
        return torch.where(z > 0, 1.0, 0.0).double()

    x = rows(s["x"])
    if c["op"] == "norm":
        g, b, du = s["gamma"].double(), s["beta"].double(), rows(s["du"])
        var, mu = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        sd = torch.sqrt(var + EPS)
        kept = eight_bits(x) if c["ckpt"] else x
        xh, a = (kept - mu) / sd, du * g
        inner = a.sum(1, keepdim=True) + xh * (a * xh).sum(1, keepdim=True)
        return {"u": back((x - mu) / sd * g + b), "u2": back(xh * g + b) if c["ckpt"] else None,
                "dx": back((a - inner / c["C"]) / sd + rows(s["skip"])), "dgamma": torch.sum(du * xh, 0), "dbeta": torch.sum(du, 0)}
    if c["op"] == "linear":
        y = act(torch.addmm(s["b"].double(), x, s["w"].double().t()))
        return back(y + rows(s["skip"]) if c["res"] else y)
    if c["op"] == "train":
        z = torch.addmm(s["b"].double(), x, s["w"].double().t())
        kept = eight_bits(z) if c["ckpt"] else z
        return {"h": back(act(z)), "z": None if c["ckpt"] else back(z), "h2": back(act(kept)), "dz": back(torch.mm(rows(s["dy"]), s["w2"].double()) * slope(kept))}
    if c["op"] == "wgrad":
        dy = rows(s["dy"])
        return {"dw": torch.mm(dy.t(), x), "db": torch.sum(dy, 0)}
    return back(eight_bits(x))
