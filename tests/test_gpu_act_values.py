"""Values at the ends of the range through the products' epilogues and the checkpoints:
infinities, NaN and the largest numbers under every activation, in every block shape."""
import math

import numpy as np
import pytest
import torch

import act_ref as R
import paper_1903_06681_amd as dc

pytestmark = pytest.mark.gpu
V = dc.View.of
INF, NAN = float("inf"), float("nan")
VALUES = [INF, -INF, NAN, 3e38, -3e38, 1e20, -1e20, 30.0, -30.0, 6.5, -6.5, 1.0, -1.0, 0.25, -0.25, 0.0]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def act(z, kind):
    """One value.  At -infinity gelu and silu are -infinity times 0, as their formulas have it: NaN."""
    if math.isnan(z) or kind == "none":
        return z
    if kind == "relu":
        return max(z, 0.0)
    if z == INF:
        return INF
    if z == -INF:
        return NAN
    if kind == "gelu":
        return z * 0.5 * math.erfc(-z / math.sqrt(2))
    return z / (1 + math.exp(-z)) if z > -700 else 0.0


# N, C, H, W, K, layout: up to 64 pixels; long sums; blocks of 64 x 64, 64 x 128 in one and two slices, 256 x 256; rows
PATHS = {"few": (1, 3, 4, 16, 40, "dense"), "few_long": (1, 300, 9, 16, 40, "dense"), "small": (2, 24, 20, 24, 72, "dense"),
         "short": (1, 24, 256, 256, 72, "dense"), "middle": (1, 72, 256, 256, 72, "dense"), "large": (1, 136, 256, 256, 256, "dense"),
         "few_row": (5, 64, 1, 1, 40, "rows"), "small_rows": (300, 64, 1, 1, 72, "rows"), "short_rows": (65536, 32, 1, 1, 64, "rows")}


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_activations_of_infinities_and_the_largest_numbers(path, dtype, out):
    """The first channel holds the value and weighs 1, the others hold zeros: z is the value."""
    N, C, H, W, K, layout = PATHS[path]
    M = N * H * W
    values = torch.tensor(VALUES).to(R.DT[dtype])
    picks = values[torch.arange(M) % len(VALUES)]
    x, _ = R.tensor(layout, N, C, H, W, dtype, fill=0.0)
    x[:, 0] = picks.view(N, H, W).cuda()
    w = torch.ones(K, C, dtype=R.DT[dtype], device="cuda")
    z, _ = R.tensor(layout, N, K, H, W, "f32")
    y, _ = R.tensor(layout, N, K, H, W, out)
    h, _ = R.tensor(layout, N, K, H, W, out)
    dz, _ = R.tensor(layout, N, K, H, W, "f32")
    dy, _ = R.tensor(layout, N, C, H, W, dtype, fill=1.0)
    w2 = torch.ones(C, K, dtype=R.DT[dtype], device="cuda")

    def compare(t, kind, what):
        got = R.f64(t).transpose(1, 0, 2).reshape(K, M)
        want = np.array([act(float(v), kind) for v in values])
        # 4e-7 |z| as elsewhere, while the tail counts; a few roundings of the value, one of them to bf16
        top = np.where(np.isfinite(want), np.abs(values.double().numpy()), 0)
        tol = 4e-7 * np.minimum(top, 10) + 2e-6 * np.abs(want) + (R.BF * np.abs(want) if out == "bf16" and what != "z" else 0)
        idx = np.arange(M) % len(VALUES)
        R.close(got, np.broadcast_to(want[idx], got.shape), tol[idx], f"{what} {kind}")

    for kind in ("none", "relu", "gelu", "silu"):
        dc.linear_fwd(V(x), x, w, None, dc.ACT[kind], None, None, V(z), z, V(y), y)
        compare(z, "none", "z")
        compare(y, kind, "y")
        if kind == "none":
            continue
        h.fill_(NAN)
        dc.linear_bwd_data(V(dy), dy, w2, dc.ACT[kind], V(z), z, V(h), h, V(dz), dz)
        compare(h, kind, "h")
        # the slope of what is finite is finite, and C at the far right, 0 at the far left
        got = R.f64(dz).transpose(1, 0, 2).reshape(K, M)
        for i, v in enumerate(values[:min(M, len(VALUES))].tolist()):
            if math.isfinite(v) and abs(v) >= 30:
                assert np.allclose(got[:, i], C if v > 0 else 0, rtol=2e-6, atol=1e-8 * C), (kind, v)


@pytest.mark.parametrize("kind", ["relu", "gelu", "silu"])
def test_checkpoint_of_the_largest_numbers_under_an_activation(kind):
    x = torch.zeros(1, 40, 1, 9)
    for p, v in enumerate((3.4e38, -3.4e38, 1e30, -1e30, 2.0 ** -126, 0.0, 100.0, -100.0, INF)):
        x[0, 0, 0, p] = v
    t, y = x.cuda(), torch.empty(1, 40, 1, 9, device="cuda")
    q = torch.empty(dc.ckpt_bytes(dc.View.q8(1, 40, 1, 9)), dtype=torch.uint8, device="cuda")
    dc.ckpt_save(V(t), t, q)
    dc.ckpt_load(dc.View.q8(1, 40, 1, 9), q, dc.ACT[kind], V(y), y)
    kept = R.q8_decode(q, 1, 40, 9)
    want = np.vectorize(lambda v: act(float(v), kind))(kept)
    R.close(R.f64(y), want, 2e-6 * np.abs(want) + 1e-30, kind)


def test_checkpoint_of_a_sample_with_more_blocks_than_32_bits_count():
    """96 channels of 2^32 / 3 pixels: a block's number passes 2^32.  Rows are one row in memory."""
    H, W = (1 << 20) + 1, 1366
    vq = dc.View.q8(1, 96, H, W)
    need, P = dc.ckpt_bytes(vq), H * W
    assert 3 * P > 1 << 32 and P < 1 << 31
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip("needs 142 GB of the card")
    g = torch.Generator()
    g.manual_seed(1)
    x = torch.randn(1, 96, 1, W, generator=g).cuda()
    q = torch.empty(need, dtype=torch.uint8, device="cuda")
    q[P * 32 * 3 - (1 << 20):P * 32 * 3].fill_(85)
    q[P * 33 * 3 - 65536:].fill_(85)
    dc.ckpt_save(V(x.expand(1, 96, H, W)), x, q)
    row = R.q8_values(R.f64(x))[0]
    scales = q[P * 32 * 3:P * 33 * 3]
    for cb in range(3):
        for first in (0, (1 << 30) - 100, (1 << 32) - 2 * P - 100, P - 2000):   # two starts, the place where the number wraps, the end
            n, at = 2000, cb * P + first
            v = q[at * 32:(at + n) * 32].view(torch.int8).view(n, 32).double()
            s = torch.exp2(scales[at:at + n].double() - 133)
            want = torch.from_numpy(row[32 * cb:32 * cb + 32]).t()[(first + torch.arange(n)) % W]
            assert torch.equal((v * s[:, None]).cpu(), want), (cb, first)
    del q, scales
    torch.cuda.empty_cache()


# every second row of an odd tile, every third channel, planes that follow a last row directly
STEPS = {"rows": lambda d: (full(d, 2, 40, 13, 18)[:, :, ::2], 2, 40, 7, 18), "channels": lambda d: (full(d, 2, 70, 6, 21)[:, ::3], 2, 24, 6, 21),
         "tight": lambda d: (torch.as_strided(full(d, 1, 1, 1, 2 * 40 * 182), (2, 40, 8, 14), (40 * 182, 182, 24, 1)), 2, 40, 8, 14)}


def full(dtype, *shape):
    return torch.full(shape, NAN, dtype=R.DT[dtype], device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", STEPS)
def test_results_in_slices_with_steps(name, dtype):
    """The same bits as in a dense result, and nothing beside them."""
    y, N, C, H, W = STEPS[name](dtype)
    base = y._base
    g = torch.Generator()
    g.manual_seed(5)
    x, w = torch.randn(N, C, H, W, generator=g).to(R.DT[dtype]).cuda(), torch.randn(C, C, generator=g).to(R.DT[dtype]).cuda()
    q = torch.empty(dc.ckpt_bytes(dc.View.q8(N, C, H, W)), dtype=torch.uint8, device="cuda")
    dc.ckpt_save(V(x), x, q)
    calls = {"norm": lambda t: dc.norm_fwd(V(x), x, None, None, 1e-5, V(t), t),
             "product": lambda t: dc.linear_fwd(V(x), x, w, None, dc.DC_ACT_GELU, None, None, None, None, V(t), t),
             "gradient": lambda t: dc.linear_bwd_data(V(x), x, w, dc.DC_ACT_NONE, None, None, None, None, V(t), t),
             "load": lambda t: dc.ckpt_load(dc.View.q8(N, C, H, W), q, dc.DC_ACT_NONE, V(t), t)}
    for what, call in calls.items():
        dense = torch.empty(N, C, H, W, dtype=R.DT[dtype], device="cuda")
        base.fill_(NAN)
        call(dense)
        call(y)
        assert torch.equal(y, dense), what
        assert R.untouched(y, base), what


def points(seed, n):
    """Normal values of several scales, dense around 0 and out to +-30."""
    g = torch.Generator()
    g.manual_seed(seed)
    z = torch.randn(5, n // 5, generator=g) * torch.tensor([0.01, 0.05, 0.3, 1.0, 8.0])[:, None]
    return z.view(-1)


def test_gelu_of_fp32_results_is_as_exact_as_fp32():
    """Bounds from the roundings.  The tail is 2^(-1 - a R(a)) within 5.3e-9; its exponential an ulp off (2^-23 of
    at most 1/2), its exponent's roundings weighed by a R 2^(-1 - a R) <= 0.27 (2^-23 of that), the sum with 1 and the
    product with z 2^-24 each: 1.6e-7 |z| with the last of them taken at Phi <= 1.  The slope: Phi once more and
    z phi(z) <= 0.25 by four operations: 4e-7."""
    z = points(3, 40000)
    x = z.view(1, 1, 100, 400).cuda()
    w, w2 = torch.ones(2, 1, device="cuda"), torch.ones(1, 2, device="cuda")
    y, h, dz, kz = (torch.empty(1, 2, 100, 400, device="cuda") for _ in range(4))
    dc.linear_fwd(V(x), x, w, None, dc.DC_ACT_GELU, None, None, V(kz), kz, V(y), y)
    assert torch.equal(kz[:, :1], x)
    dy = torch.ones(1, 1, 100, 400, device="cuda")
    dc.linear_bwd_data(V(dy), dy, w2, dc.DC_ACT_GELU, V(kz), kz, V(h), h, V(dz), dz)
    zd = z.double()
    want = zd * torch.special.ndtr(zd)
    slope = torch.special.ndtr(zd) + zd * torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi)
    for t, what in ((y, "y"), (h, "h")):
        R.close(R.f64(t)[0, 0], want.numpy(), 1.6e-7 * zd.abs().numpy(), what)
        assert torch.equal(t[:, 0], t[:, 1])
    R.close(R.f64(dz)[0, 0], slope.numpy(), 4e-7, "slope")
    assert torch.equal(h, y)
    # at small scales the root of the mean square error stays within a rounding and a half of the values'
    small = (zd.abs() < 0.3) & (zd != 0)
    err = (y[0, 0].cpu().double().view(-1) - want)[small]
    assert float(err.norm() / want[small].norm()) < 1.5 * R.EPS32
