"""Python binding of libdc: one GPU's share of a spatially decomposed 2-D
convolution layer (Dryden et al., arXiv 1903.06681) on MI355X.

Argument marshalling only.  Every step of the computation runs in the HIP
kernels behind the C ABI declared in ``include/dc.h``; this module converts
torch tensors to device pointers, passes the current HIP stream and turns a
negative status into an exception.  There is no CPU fallback: importing the
package fails if ``libdc.so`` has not been built.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdc.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build the HIP library first "
        "(python -c 'import __graft_entry__ as g; g.build()')")

# torch brings its own HIP runtime (same soname as /opt/rocm's).  Loading it
# first makes libdc.so bind to that one copy: with the library loaded first,
# the process would hold two runtimes, and pointers and streams from torch
# would be foreign to the library's launches.
import torch  # noqa: E402,F401

_lib = ctypes.CDLL(LIB_PATH)

DC_F32, DC_BF16 = 0, 1
DC_X, DC_DY = 0, 1
DC_ALL_TILES = -1
DC_BAND_NS, DC_BAND_WE, DC_BAND_CORNERS, DC_BAND_ALL = 1, 2, 4, 7
DC_REGION_ALL, DC_REGION_INTERIOR, DC_REGION_BOUNDARY = 0, 1, 2
DC_Q8 = 2   # view dtype: an activation checkpoint in 8 bits
DC_ACT_NONE, DC_ACT_RELU, DC_ACT_GELU, DC_ACT_SILU = 0, 1, 2, 3
DC_NORM_NONE, DC_NORM_LAYER, DC_NORM_RMS = 0, 1, 2
NORM = {"none": DC_NORM_NONE, "layer": DC_NORM_LAYER, "rms": DC_NORM_RMS}
ACT = {"none": DC_ACT_NONE, "relu": DC_ACT_RELU, "gelu": DC_ACT_GELU, "silu": DC_ACT_SILU}
# capacity of the fixed workspace of dc_conv_bwd_filter_noalloc (include/dc.h)
BWD_FILTER_NOALLOC_MAX_BYTES = 64 << 20

STATUS = {
    0: "DC_OK", -1: "DC_ERR_NULL", -2: "DC_ERR_SHAPE", -3: "DC_ERR_DTYPE", -4: "DC_ERR_HALO",
    -5: "DC_ERR_UNSUPPORTED", -6: "DC_ERR_WORKSPACE", -7: "DC_ERR_ALIGN", -8: "DC_ERR_HIP",
    -9: "DC_ERR_TILE", -10: "DC_ERR_ARG", -11: "DC_ERR_TOO_LARGE",
}

EXPORTS = (
    "dc_conv_fwd", "dc_conv_bwd_data", "dc_conv_bwd_filter", "dc_halo_pack", "dc_halo_unpack",
    "dc_conv_bwd_filter_noalloc", "dc_halo_pack_bands", "dc_halo_unpack_bands",
    "dc_conv_fwd_region", "dc_conv_bwd_data_region", "dc_validate",
    "dc_tile_pitch", "dc_tile_elems", "dc_halo_elems", "dc_bwd_filter_workspace_bytes",
    "dc_required_halo", "dc_halo_bands", "dc_tile_dims", "dc_status_string",
    "dc_ckpt_bytes", "dc_ckpt_save", "dc_ckpt_load", "dc_norm_fwd", "dc_norm_bwd", "dc_norm_bwd_workspace_bytes",
    "dc_linear_fwd", "dc_linear_bwd_data", "dc_linear_bwd_filter", "dc_linear_bwd_filter_workspace_bytes",
    "dc_dropout", "dc_gate_fwd", "dc_gate_bwd_data", "dc_join_fwd", "dc_join_bwd", "dc_join_bwd_workspace_bytes",
)


class Problem(ctypes.Structure):
    """``dc_problem``: the layer (Sec. II-A) and its P x Q blocked grid (Sec. III-A)."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("N", "C", "K", "H", "W", "R", "S", "stride", "pad", "P", "Q", "halo", "dtype")]

    @classmethod
    def of(cls, layer) -> "Problem":
        """From any object with the same field names (dtype 'f32'/'bf16' or int)."""
        dt = layer.dtype
        if isinstance(dt, str):
            dt = {"f32": DC_F32, "bf16": DC_BF16}[dt]
        return cls(layer.N, layer.C, layer.K, layer.H, layer.W, layer.R, layer.S,
                   layer.stride, layer.pad, layer.P, layer.Q, layer.halo, dt)


_VIEW_DT = {torch.float32: DC_F32, torch.bfloat16: DC_BF16}


class View(ctypes.Structure):
    """``dc_view``: a tensor [N][C][H][W] in memory, columns contiguous.

    Built once per layout (``of`` a tensor, ``q8`` for a checkpoint) and passed
    beside the tensor it describes.
    """
    _fields_ = ([(n, ctypes.c_int32) for n in ("N", "C", "H", "W")] +
                [(n, ctypes.c_int64) for n in ("sn", "sc", "sh")] + [("dtype", ctypes.c_int32)])

    @classmethod
    def of(cls, t) -> "View":
        """Of a 4-D fp32 or bf16 tensor, or slice of one, whose columns are contiguous."""
        if t.dim() != 4 or t.dtype not in _VIEW_DT:
            raise ValueError(f"a view describes a 4-D float32 or bfloat16 tensor, not {t.dim()}-D {t.dtype}")
        (n, c, h, w), (sn, sc, sh, sw) = t.shape, t.stride()
        if sw != 1 and w > 1:
            raise ValueError(f"a view's columns are contiguous: got a column stride of {sw}")
        return cls(n, c, h, w, sn, sc, sh, _VIEW_DT[t.dtype])

    @classmethod
    def q8(cls, N, C, H, W) -> "View":
        """Of the 8-bit checkpoint of such a tensor (a buffer of ckpt_bytes)."""
        return cls(N, C, H, W, 0, 0, 0, DC_Q8)


class Drop(ctypes.Structure):
    """``dc_drop``: a dropout whose mask is formed again wherever it is read.

    p: the share that is dropped; seed and offset (an offset of its own for each use) choose
    the mask; step: a CUDA int64 or uint64 tensor of one element that is added to the offset
    when the kernel runs, or None.  n0, h0, w0, H, W, P, Q: where the tensor lies in the whole
    one (a tile in its image; 0: the tensor is the whole).
    """
    _fields_ = ([("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("step", ctypes.c_void_p)] +
                [(n, ctypes.c_int32) for n in ("n0", "h0", "w0", "H", "W", "P", "Q")])

    def __init__(self, p, seed, offset=0, step=None, n0=0, h0=0, w0=0, H=0, W=0, P=0, Q=0):
        super().__init__(p, seed, offset, _ptr(step), n0, h0, w0, H, W, P, Q)
        self._step = step                     # alive as long as its address is


class Norm(ctypes.Structure):
    """``dc_norm``: a norm over a pixel's channels; gamma and beta are fp32 tensors or None."""
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("_gamma", ctypes.c_void_p), ("_beta", ctypes.c_void_p)]

    def __init__(self, kind, eps, gamma=None, beta=None):
        super().__init__(kind, eps, _ptr(gamma), _ptr(beta))
        self.gamma, self.beta = gamma, beta


class JoinGrads(ctypes.Structure):
    """``dc_join_grads``: where join_bwd writes the parameters' gradients (fp32 tensors or None)."""
    _names = ("scale", "gate", "gamma_post", "beta_post", "gamma_pre", "beta_pre")
    _fields_ = [("_" + n, ctypes.c_void_p) for n in _names]

    def __init__(self, scale=None, gate=None, gamma_post=None, beta_post=None, gamma_pre=None, beta_pre=None):
        t = (scale, gate, gamma_post, beta_post, gamma_pre, beta_pre)
        super().__init__(*map(_ptr, t))
        self.scale, self.gate, self.gamma_post, self.beta_post, self.gamma_pre, self.beta_pre = t


class DcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} "
                         f"({_lib.dc_status_string(status).decode()})")


_P = ctypes.POINTER(Problem)
_V = ctypes.c_void_p
_I = ctypes.c_int32
_lib.dc_conv_fwd.argtypes = [_P, _I, _V, _V, _V, _V]
_lib.dc_conv_bwd_data.argtypes = [_P, _I, _V, _V, _V, _V]
_lib.dc_conv_bwd_filter.argtypes = [_P, _I, _V, _V, _V, _I, _V, ctypes.c_size_t, _V]
_lib.dc_conv_bwd_filter_noalloc.argtypes = [_P, _I, _V, _V, _V, _I, _V]
_lib.dc_halo_pack.argtypes = [_P, _I, _I, _V, _V, _V]
_lib.dc_halo_unpack.argtypes = [_P, _I, _I, _V, _V, _V]
_lib.dc_conv_fwd_region.argtypes = [_P, _I, _I, _V, _V, _V, _V]
_lib.dc_conv_bwd_data_region.argtypes = [_P, _I, _I, _V, _V, _V, _V]
_lib.dc_halo_pack_bands.argtypes = [_P, _I, _I, _I, _V, _V, _V]
_lib.dc_halo_unpack_bands.argtypes = [_P, _I, _I, _I, _V, _V, _V]
_lib.dc_halo_bands.argtypes = [_P, _I, ctypes.POINTER(_I)]
_lib.dc_validate.argtypes = [_P, _I]
_lib.dc_tile_pitch.argtypes = [_P, _I]
_lib.dc_tile_pitch.restype = ctypes.c_int64
_lib.dc_tile_elems.argtypes = [_P, _I]
_lib.dc_tile_elems.restype = ctypes.c_int64
_lib.dc_halo_elems.argtypes = [_P, _I]
_lib.dc_halo_elems.restype = ctypes.c_int64
_lib.dc_bwd_filter_workspace_bytes.argtypes = [_P, _I]
_lib.dc_bwd_filter_workspace_bytes.restype = ctypes.c_size_t
_lib.dc_required_halo.argtypes = [_P, _I, ctypes.POINTER(_I)]
_lib.dc_tile_dims.argtypes = [_P, ctypes.POINTER(_I)]
_lib.dc_status_string.argtypes = [_I]
_lib.dc_status_string.restype = ctypes.c_char_p
_W = ctypes.POINTER(View)
_Z = ctypes.c_size_t
_lib.dc_ckpt_bytes.argtypes = [_W]
_lib.dc_ckpt_bytes.restype = ctypes.c_int64
_lib.dc_ckpt_save.argtypes = [_W, _V, _V, _V]
_lib.dc_ckpt_load.argtypes = [_W, _V, _I, _W, _V, _V]
_lib.dc_norm_fwd.argtypes = [_W, _V, _V, _V, ctypes.c_float, _W, _V, _V, _V, _V]
_lib.dc_norm_bwd.argtypes = [_W, _V, _W, _V, _V, _V, _V, _W, _V, _W, _V, _W, _V, _V, _V, _I, _V, _Z, _V]
_lib.dc_norm_bwd_workspace_bytes.argtypes = [_W]
_lib.dc_norm_bwd_workspace_bytes.restype = _Z
_lib.dc_linear_fwd.argtypes = [_W, _V, _V, _V, _I, _W, _V, _W, _V, _W, _V, _V]
_lib.dc_linear_bwd_data.argtypes = [_W, _V, _V, _I, _W, _V, _W, _V, _W, _V, _V]
_lib.dc_linear_bwd_filter.argtypes = [_W, _V, _W, _V, _V, _V, _I, _V, _Z, _V]
_lib.dc_linear_bwd_filter_workspace_bytes.argtypes = [_W, _W]
_lib.dc_linear_bwd_filter_workspace_bytes.restype = _Z
_D, _N, _G = ctypes.POINTER(Drop), ctypes.POINTER(Norm), ctypes.POINTER(JoinGrads)
_lib.dc_dropout.argtypes = [_D, _W, _V, _W, _V, _V]
_lib.dc_gate_fwd.argtypes = [_W, _V, _V, _V, _I, _D, _W, _V, _V, _W, _V, _V]
_lib.dc_gate_bwd_data.argtypes = [_W, _V, _V, _I, _D, _W, _V, _V, _W, _V, _W, _V, _V]
_lib.dc_join_fwd.argtypes = [_W, _V, _N, _V, _V, _D, _W, _V, _N, _W, _V, _W, _V, _V, _V, _V]
_lib.dc_join_bwd.argtypes = [_W, _V, _W, _V, _W, _V, _W, _V, _W, _V, _V, _N, _V, _V, _D, _N, _W, _V, _W, _V, _G, _I, _V, _Z, _V]
_lib.dc_join_bwd_workspace_bytes.argtypes = [_W, _I]
_lib.dc_join_bwd_workspace_bytes.restype = _Z
for _n in ("dc_ckpt_save", "dc_ckpt_load", "dc_norm_fwd", "dc_norm_bwd", "dc_linear_fwd", "dc_linear_bwd_data",
           "dc_linear_bwd_filter", "dc_dropout", "dc_gate_fwd", "dc_gate_bwd_data", "dc_join_fwd", "dc_join_bwd"):
    getattr(_lib, _n).restype = ctypes.c_int32
for _n in ("dc_conv_fwd", "dc_conv_bwd_data", "dc_conv_bwd_filter", "dc_conv_bwd_filter_noalloc",
           "dc_halo_pack", "dc_halo_unpack", "dc_halo_pack_bands", "dc_halo_unpack_bands",
           "dc_conv_fwd_region", "dc_conv_bwd_data_region",
           "dc_validate", "dc_required_halo", "dc_halo_bands", "dc_tile_dims"):
    getattr(_lib, _n).restype = ctypes.c_int32


def lib():
    return _lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# The current stream's handle without building a Stream object: a call of a
# small layer takes 7 us on the host, 2.8 of them in current_stream().  torch
# keeps one current stream per device; builds without these two bindings (or
# without a GPU) take the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(st, where):
    if st != 0:
        raise DcError(st, where)


# ---------------------------------------------------------------- host helpers

def validate(prob: Problem, tile: int = DC_ALL_TILES) -> int:
    return _lib.dc_validate(ctypes.byref(prob), tile)


def tile_pitch(prob, which):
    return _lib.dc_tile_pitch(ctypes.byref(prob), which)


def tile_elems(prob, which):
    return _lib.dc_tile_elems(ctypes.byref(prob), which)


def halo_elems(prob, which):
    return _lib.dc_halo_elems(ctypes.byref(prob), which)


def bwd_filter_workspace_bytes(prob, tile):
    return _lib.dc_bwd_filter_workspace_bytes(ctypes.byref(prob), tile)


def required_halo(prob, which):
    out = (_I * 2)()
    _check(_lib.dc_required_halo(ctypes.byref(prob), which, out), "dc_required_halo")
    return out[0], out[1]


def halo_bands(prob, which):
    """Band widths (above, below, left, right) the halo calls move for x or dy."""
    out = (_I * 4)()
    _check(_lib.dc_halo_bands(ctypes.byref(prob), which, out), "dc_halo_bands")
    return tuple(out)


def tile_dims(prob):
    out = (_I * 4)()
    _check(_lib.dc_tile_dims(ctypes.byref(prob), out), "dc_tile_dims")
    return tuple(out)


def tile_shape(prob, which):
    """Shape [N, channels, rows + 2h, pitch] of one padded tile."""
    Ht, Wt, Hot, Wot = tile_dims(prob)
    ch = prob.C if which == DC_X else prob.K
    rows = (Ht if which == DC_X else Hot) + 2 * prob.halo
    return (prob.N, ch, rows, tile_pitch(prob, which))


# ---------------------------------------------------------------- the five calls

def conv_fwd(prob, tile, x_pad, w, y, stream=None):
    """Eq. (1) on a tile: y <- conv(x_pad, w)."""
    _check(_lib.dc_conv_fwd(ctypes.byref(prob), tile, _ptr(x_pad), _ptr(w), _ptr(y),
                            _stream(stream)), "dc_conv_fwd")


def conv_bwd_data(prob, tile, dy_pad, w, dx, stream=None):
    """Eq. (3) on a tile: dx <- input gradient from dy_pad and w."""
    _check(_lib.dc_conv_bwd_data(ctypes.byref(prob), tile, _ptr(dy_pad), _ptr(w), _ptr(dx),
                                 _stream(stream)), "dc_conv_bwd_data")


def conv_bwd_filter(prob, tile, x_pad, dy_pad, dw, accumulate, workspace, stream=None):
    """Eq. (2) on a tile: dw (=|+=) local weight gradient."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.dc_conv_bwd_filter(ctypes.byref(prob), tile, _ptr(x_pad), _ptr(dy_pad),
                                   _ptr(dw), accumulate, _ptr(workspace), ws_bytes,
                                   _stream(stream)), "dc_conv_bwd_filter")


def conv_bwd_filter_noalloc(prob, tile, x_pad, dy_pad, dw, accumulate, stream=None):
    """Eq. (2) on a tile with the library's fixed device workspace (no allocation)."""
    _check(_lib.dc_conv_bwd_filter_noalloc(ctypes.byref(prob), tile, _ptr(x_pad), _ptr(dy_pad),
                                           _ptr(dw), accumulate, _stream(stream)),
           "dc_conv_bwd_filter_noalloc")


def halo_pack(prob, tile, which, t_pad, send, stream=None):
    """Copy the bands neighbours need into the packed send buffer."""
    _check(_lib.dc_halo_pack(ctypes.byref(prob), tile, which, _ptr(t_pad), _ptr(send),
                             _stream(stream)), "dc_halo_pack")


def halo_unpack(prob, tile, which, recv, t_pad, stream=None):
    """Fill the margins of t_pad from the receive buffer (zeros at the domain edge)."""
    _check(_lib.dc_halo_unpack(ctypes.byref(prob), tile, which, _ptr(recv), _ptr(t_pad),
                               _stream(stream)), "dc_halo_unpack")


def halo_pack_bands(prob, tile, which, bands, t_pad, send, stream=None):
    """halo_pack restricted to the DC_BAND_* classes in `bands`."""
    _check(_lib.dc_halo_pack_bands(ctypes.byref(prob), tile, which, bands, _ptr(t_pad), _ptr(send),
                                   _stream(stream)), "dc_halo_pack_bands")


def halo_unpack_bands(prob, tile, which, bands, recv, t_pad, stream=None):
    """halo_unpack restricted to the DC_BAND_* classes in `bands`."""
    _check(_lib.dc_halo_unpack_bands(ctypes.byref(prob), tile, which, bands, _ptr(recv), _ptr(t_pad),
                                     _stream(stream)), "dc_halo_unpack_bands")


def conv_fwd_region(prob, tile, region, x_pad, w, y, stream=None):
    """Eq. (1) on the interior (no halo read) or the boundary frame of a tile."""
    _check(_lib.dc_conv_fwd_region(ctypes.byref(prob), tile, region, _ptr(x_pad), _ptr(w), _ptr(y),
                                   _stream(stream)), "dc_conv_fwd_region")


def conv_bwd_data_region(prob, tile, region, dy_pad, w, dx, stream=None):
    """Eq. (3) on the interior (no halo read) or the boundary frame of a tile."""
    _check(_lib.dc_conv_bwd_data_region(ctypes.byref(prob), tile, region, _ptr(dy_pad), _ptr(w),
                                        _ptr(dx), _stream(stream)), "dc_conv_bwd_data_region")


# ------------------------------------- between two convolutions (views: View)

def _view(v):
    return None if v is None else ctypes.byref(v)


def _bytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def ckpt_bytes(vq):
    """Bytes of the 8-bit checkpoint of a tensor of vq's N, C, H, W; -1 if invalid."""
    return _lib.dc_ckpt_bytes(ctypes.byref(vq))


def ckpt_save(vx, x, q, stream=None):
    """q <- x in 8 bits."""
    _check(_lib.dc_ckpt_save(_view(vx), _ptr(x), _ptr(q), _stream(stream)), "dc_ckpt_save")


def ckpt_load(vq, q, act, vy, y, stream=None):
    """y <- act(what q stands for)."""
    _check(_lib.dc_ckpt_load(_view(vq), _ptr(q), act, _view(vy), _ptr(y), _stream(stream)), "dc_ckpt_load")


def norm_fwd(vx, x, gamma, beta, eps, vu, u, stat=None, ckpt=None, stream=None):
    """u <- layer norm of each pixel of x over its channels; stat (mean, 1/deviation) and
    ckpt (x in 8 bits) for the backward pass."""
    _check(_lib.dc_norm_fwd(_view(vx), _ptr(x), _ptr(gamma), _ptr(beta), eps, _view(vu), _ptr(u), _ptr(stat),
                            _ptr(ckpt), _stream(stream)), "dc_norm_fwd")


def norm_bwd_workspace_bytes(vdu):
    return _lib.dc_norm_bwd_workspace_bytes(ctypes.byref(vdu))


def norm_bwd(vdu, du, vx, x, stat, gamma, beta, vres, res, vu, u, vdx, dx, dgamma, dbeta, accumulate, workspace,
             stream=None):
    """dx <- input gradient of norm_fwd (+ res), dgamma, dbeta (=|+=) the parameters'; x is the
    input or its checkpoint (vx of dtype DC_Q8).  res, u (the forward's output again), dgamma and
    dbeta may be None."""
    _check(_lib.dc_norm_bwd(_view(vdu), _ptr(du), _view(vx), _ptr(x), _ptr(stat), _ptr(gamma), _ptr(beta),
                            _view(vres), _ptr(res), _view(vu), _ptr(u), _view(vdx), _ptr(dx), _ptr(dgamma),
                            _ptr(dbeta), accumulate, _ptr(workspace), _bytes(workspace), _stream(stream)),
           "dc_norm_bwd")


def linear_fwd(vx, x, w, bias, act, vres, res, vz, z, vy, y, stream=None):
    """y <- act(w x + bias) + res over the channels of every pixel; z (whole or 8-bit) keeps what
    act reads.  bias, res and z may be None."""
    _check(_lib.dc_linear_fwd(_view(vx), _ptr(x), _ptr(w), _ptr(bias), act, _view(vres), _ptr(res), _view(vz),
                              _ptr(z), _view(vy), _ptr(y), _stream(stream)), "dc_linear_fwd")


def linear_bwd_data(vdy, dy, w, act, vz, z, vh, h, vdx, dx, stream=None):
    """dx <- (w^T dy) act'(z); h <- act(z) again unless None.  act DC_ACT_NONE: z and h are None."""
    _check(_lib.dc_linear_bwd_data(_view(vdy), _ptr(dy), _ptr(w), act, _view(vz), _ptr(z), _view(vh), _ptr(h),
                                   _view(vdx), _ptr(dx), _stream(stream)), "dc_linear_bwd_data")


def linear_bwd_filter_workspace_bytes(vx, vdy):
    return _lib.dc_linear_bwd_filter_workspace_bytes(ctypes.byref(vx), ctypes.byref(vdy))


def linear_bwd_filter(vx, x, vdy, dy, dw, db, accumulate, workspace, stream=None):
    """dw (=|+=) sum over pixels of dy x^T, db (=|+=) sum over pixels of dy (or None)."""
    _check(_lib.dc_linear_bwd_filter(_view(vx), _ptr(x), _view(vdy), _ptr(dy), _ptr(dw), _ptr(db), accumulate,
                                     _ptr(workspace), _bytes(workspace), _stream(stream)), "dc_linear_bwd_filter")


# ------------------------------------- a gated residual block

def dropout(drop, vx, x, vy, y, stream=None):
    """y <- x dropped out (drop: Drop); the same call on dy is its gradient."""
    _check(_lib.dc_dropout(_view(drop), _view(vx), _ptr(x), _view(vy), _ptr(y), _stream(stream)), "dc_dropout")


def gate_fwd(vx, x, w, bias, act, drop, vz, zg, zu, vh, h, stream=None):
    """h <- drop(act(zg) zu), zg and zu the products of x with w's first and second half; bias,
    drop, and zg with zu (whole or 8-bit, kept for gate_bwd_data) may be None."""
    _check(_lib.dc_gate_fwd(_view(vx), _ptr(x), _ptr(w), _ptr(bias), act, _view(drop), _view(vz), _ptr(zg), _ptr(zu),
                            _view(vh), _ptr(h), _stream(stream)), "dc_gate_fwd")


def gate_bwd_data(vdy, dy, w, act, drop, vz, zg, zu, vh, h, vdz, dz, stream=None):
    """dz <- gradient at zg and zu (2 K channels) from dy, the gradient of the product w after the
    gated one; h <- drop(act(zg) zu) again unless None."""
    _check(_lib.dc_gate_bwd_data(_view(vdy), _ptr(dy), _ptr(w), act, _view(drop), _view(vz), _ptr(zg), _ptr(zu),
                                 _view(vh), _ptr(h), _view(vdz), _ptr(dz), _stream(stream)), "dc_gate_bwd_data")


def join_fwd(vy, y, post, scale, gate, drop, vx, x, pre, vo, o, vu, u, stat=None, ckpt=None, stream=None):
    """o <- x + scale gate drop(post(y)), u <- pre(o) (post, pre: Norm or None); stat [4][N][H][W]
    and ckpt (o in 8 bits) for the backward pass."""
    _check(_lib.dc_join_fwd(_view(vy), _ptr(y), _view(post), _ptr(scale), _ptr(gate), _view(drop), _view(vx), _ptr(x),
                            _view(pre), _view(vo), _ptr(o), _view(vu), _ptr(u), _ptr(stat), _ptr(ckpt), _stream(stream)),
           "dc_join_fwd")


def join_bwd_workspace_bytes(vdy, gate):
    return _lib.dc_join_bwd_workspace_bytes(ctypes.byref(vdy), int(bool(gate)))


def join_bwd(vdu, du, vdo, do, vy, y, vx, x, vo, o, stat, post, scale, gate, drop, pre, vdx, dx, vdy, dy, grads,
             accumulate, workspace, stream=None):
    """dx, dy <- gradients of join_fwd at x and y from those at u and o; grads (JoinGrads or None)
    (=|+=) the parameters'.  o is formed again from y and x, or read where it is given; the three
    are whole or their 8-bit forms."""
    _check(_lib.dc_join_bwd(_view(vdu), _ptr(du), _view(vdo), _ptr(do), _view(vy), _ptr(y), _view(vx), _ptr(x),
                            _view(vo), _ptr(o), _ptr(stat), _view(post), _ptr(scale), _ptr(gate), _view(drop), _view(pre), _view(vdx),
                            _ptr(dx), _view(vdy), _ptr(dy), _view(grads), accumulate, _ptr(workspace),
                            _bytes(workspace), _stream(stream)), "dc_join_bwd")
