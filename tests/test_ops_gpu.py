"""The operators around the step against plain implementations in 64 bits.

The bounds follow from the arithmetic, with u = 2^-24 the rounding of fp32
and 2^-8 that of bf16, and are stated at each check: how many
roundings a sum can have passed through (a thread's chain, the warp's tree,
the joined warps), relative to the sum of its terms' magnitudes.
"""
import math

import pytest
import torch

from paper_2607_01455_gb300 import Ops
from paper_2607_01455_gb300 import ember as E

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
TINY = 2.0 ** -126  # below it the relative bounds of normal numbers end


@pytest.fixture(scope="module")
def ops(cuda_device):
    return Ops(cuda_device)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def out_u(dtype):
    return 2.0 ** -8 if dtype == BF else U


def rows(g, T, D, dtype, pad=0, offset=0, scale=1.0):
    """T rows of D values as a slice of wider rows, off the 16-byte boundaries with an odd offset."""
    b = (randn(g, T, D + pad + offset) * scale).to(dtype)
    return b[:, offset:offset + D]


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    if not got.numel():
        return
    err = (got - want).abs() - bound - TINY
    assert not torch.isnan(err).any(), what
    assert err.max().item() <= 0, (what, err.max().item(), int(err.argmax()))


# ---- the norm ----

def norm64(x, gain, res, eps):
    s = x.double() if res is None else x.double() + res.double()
    n = torch.sqrt(s.square().mean(1, keepdim=True) + eps)
    return s, s / n * (1.0 if gain is None else gain.double())


# the sum of squares: up to 32 terms in a thread, 5 shuffles, 32 warps, the
# division, eps; the root halves it; then the root, the reciprocal, two
# products and the rounding of the sum itself
NORM_U = (32 + 5 + 32 + 2) / 2 * U + 6 * U

NORM_SHAPES = [(1, 1), (1, 7), (3, 8), (2, 64), (5, 65), (4, 1000), (1, 4096), (160, 4096), (153, 2048), (7, 1003),
               (9, 4099), (2, 8192), (300, 8200), (3, 16384), (2, 32768), (2, 32767), (0, 64)]


@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("xt,rt,gt", [(BF, None, F32), (BF, BF, BF), (BF, F32, F32), (F32, BF, BF), (F32, F32, F32),
                                      (F32, None, None)])
def test_norm(ops, T, D, xt, rt, gt):
    g = gen(T * 131 + D)
    x = rows(g, T, D, xt)
    res = None if rt is None else rows(g, T, D, rt, scale=3.0)
    gain = None if gt is None else (1 + 0.1 * randn(g, D)).to(gt)
    y, h = ops.rmsnorm(x, gain, residual=res, eps=1e-5)
    s64, y64 = norm64(x, gain, res, 1e-5)
    close(y, y64, (NORM_U + out_u(xt)) * y64.abs(), "y")
    if res is None:
        assert h is None
    else:
        assert h.dtype == rt
        close(h, s64, (U + out_u(rt)) * s64.abs(), "h")


@pytest.mark.parametrize("D", [64, 96, 1003, 4096])
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 3), (8, 8)])
def test_norm_of_strided_rows(ops, D, pad, offset):
    g = gen(D + pad)
    for xt in (BF, F32):
        x, res = rows(g, 33, D, xt, pad, offset), rows(g, 33, D, F32, pad, offset)
        gain = randn(g, D + offset)[offset:]
        guard = torch.full((33, D + 4), 7.0, device="cuda", dtype=xt)
        ho = torch.full((33, D + 6), 7.0, device="cuda")
        y, h = ops.rmsnorm(x, gain, residual=res, out=guard[:, 1:D + 1], residual_out=ho[:, 2:D + 2])
        s64, y64 = norm64(x, gain, res, 1e-6)
        close(y, y64, (NORM_U + out_u(xt)) * y64.abs(), "y")
        close(h, s64, 2 * U * s64.abs(), "h")
        assert (guard[:, 0] == 7).all() and (guard[:, D + 1:] == 7).all()
        assert (ho[:, :2] == 7).all() and (ho[:, D + 2:] == 7).all()


@pytest.mark.parametrize("T,D", [(1, 256), (40, 4096), (5, 33)])
def test_norm_in_place(ops, T, D):
    g = gen(5)
    x, res = rows(g, T, D, BF), rows(g, T, D, BF)
    y, h = ops.rmsnorm(x, None, residual=res)
    x2, r2 = x.clone(), res.clone()
    ops.rmsnorm(x2, None, residual=r2, out=x2, residual_out=r2)
    assert torch.equal(x2, y) and torch.equal(r2, h)


def test_norm_of_zero_infinite_and_nan_rows(ops):
    x = randn(gen(1), 6, 512)
    x[0] = 0
    x[1, 3] = math.inf
    x[2, 4] = math.nan
    x[3] *= 1e-30
    x[4] *= 1e-42  # subnormal
    y, _ = ops.rmsnorm(x, None, eps=1e-6)
    assert (y[0] == 0).all()
    assert torch.isnan(y[1, 3]) and (y[1, :3] == 0).all() and (y[1, 4:] == 0).all()
    assert torch.isnan(y[2]).all()
    y64 = norm64(x, None, None, 1e-6)[1]
    close(y[3:], y64[3:], NORM_U * y64[3:].abs() + U * TINY, "small rows")
    y, _ = ops.rmsnorm(torch.zeros(2, 64, device="cuda"), None, eps=0.0)
    assert torch.isnan(y).all()  # 0 / 0, as the formula has it
    q, s, _ = ops.rmsnorm_quant(x, None, eps=1e-6)
    assert s[0] == 0 and (q[0] == 0).all()
    assert torch.isnan(s[1:3]).all() and (q[1:3] == 0).all()


def check_rows8(q, scales, y64, rel):
    """scales = max |y| / 127 and q within a half (and what a relative error
    `rel` of y and scale does at 127) of y / scale."""
    top = y64.abs().amax(1)
    close(scales, top / 127, (rel + 2 * U) * top / 127, "scales")
    ideal = y64 / (top / 127).clamp(min=1e-300)[:, None]
    assert ((q.double() - ideal).abs() <= 0.5 + 127 * (2 * rel + 4 * U)).all()
    assert q.dtype == torch.int8 and (q.abs() <= 127).all() and (q != -128).all()


@pytest.mark.parametrize("T,D", [(1, 1), (3, 7), (2, 64), (5, 1003), (160, 4096), (9, 8200), (2, 32768), (0, 16)])
@pytest.mark.parametrize("xt,rt", [(BF, None), (BF, BF), (F32, F32), (F32, None)])
def test_norm_in_8_bits(ops, T, D, xt, rt):
    g = gen(T + D)
    x = rows(g, T, D, xt)
    res = None if rt is None else rows(g, T, D, rt)
    gain = 1 + 0.1 * randn(g, D)
    q, scales, h = ops.rmsnorm_quant(x, gain, residual=res)
    s64, y64 = norm64(x, gain, res, 1e-6)
    if T:
        check_rows8(q, scales, y64, NORM_U)
    if res is not None:
        close(h, s64, (U + out_u(rt)) * s64.abs(), "h")
    back = ops.dequantize_rows(q, scales, dtype=F32)
    assert torch.equal(back, q.float() * scales[:, None])
    assert torch.equal(ops.dequantize_rows(q, scales), back.to(BF))


@pytest.mark.parametrize("T,D,pad", [(1, 1, 0), (7, 64, 0), (200, 1003, 0), (33, 96, 5), (1000, 768, 0), (3, 32768, 0)])
@pytest.mark.parametrize("xt", [BF, F32])
def test_quantize_rows(ops, T, D, pad, xt):
    x = rows(gen(D), T, D, xt, pad) * torch.logspace(-30, 30, T, device="cuda")[:, None].to(xt)
    q, scales = ops.quantize_rows(x)
    assert q.stride(0) % 16 == 0
    check_rows8(q, scales, x.double(), 0.0)


def test_quantize_rows_of_tiny_and_empty(ops):
    x = torch.zeros(4, 48, device="cuda")
    x[1, 5] = 1e-40
    x[2] = torch.linspace(-2e-36, 2e-36, 48, device="cuda")
    x[3] = torch.finfo(F32).max
    q, s = ops.quantize_rows(x)
    assert s[0] == 0 and (q[0] == 0).all()
    assert 120 <= q[1, 5] <= 127 and (q[1].bool().sum() == 1)  # a subnormal scale has few bits
    assert ((q[2].double() - x[2].double() / (2e-36 / 127)).abs() <= 0.51).all()
    assert (q[3] == 127).all()
    q, s = ops.quantize_rows(torch.empty(0, 48, device="cuda"))
    assert q.shape == (0, 48) and s.shape == (0,)


# ---- the norm's gradients ----

def back64(dy, h, gain, eps, dres):
    h, dy = h.double(), dy.double()
    D = h.shape[1]
    n = torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    a = dy if gain is None else dy * gain.double()
    c = (a * h).sum(1, keepdim=True) / (D * n ** 3)
    dx = a / n - h * c
    mag = (a / n).abs() + h.abs() * (a * h).abs().sum(1, keepdim=True) / (D * n ** 3)
    if dres is not None:
        dx = dx + dres.double()
        mag = mag + dres.double().abs()
    return dx, mag, (dy * h / n).sum(0), (dy * h / n).abs().sum(0)


# n^3: three times the norm's error; the dot's chain of up to 32 + 5 + 32
BACK_U = 3 * NORM_U + 80 * U

BACK_SHAPES = [(1, 1), (1, 64), (3, 7), (700, 64), (17, 1003), (2500, 1003), (33, 2048), (310, 4096), (5, 5000),
               (1300, 8192), (40, 16384), (3, 32768), (2, 20001), (2, 4097), (0, 32)]


@pytest.mark.parametrize("T,D", BACK_SHAPES)
@pytest.mark.parametrize("t,gt,with_dres", [(BF, F32, True), (BF, BF, False), (F32, F32, False), (F32, BF, True),
                                            (F32, None, False)])
def test_norm_backward(ops, T, D, t, gt, with_dres):
    g = gen(T * 7 + D)
    h, dy = rows(g, T, D, t, scale=2.0), rows(g, T, D, t, scale=1e-3)
    dres = rows(g, T, D, t, scale=1e-3) if with_dres else None
    gain = None if gt is None else (1 + 0.1 * randn(g, D)).to(gt)
    dx, dgain = ops.rmsnorm_backward(dy, h, gain, eps=1e-5, dres=dres)
    dx64, mag, dg64, dgmag = back64(dy, h, gain, 1e-5, dres)
    close(dx, dx64, BACK_U * mag + out_u(t) * dx64.abs(), "dx")
    # every row's term, then at most T additions
    close(dgain, dg64, (T + 8) * U * dgmag + NORM_U * dgmag, "dgain")


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (8, 8)])
@pytest.mark.parametrize("D", [64, 1003, 4096])
def test_norm_backward_of_strided_rows(ops, D, pad, offset):
    g = gen(D)
    h, dy, dres = (rows(g, 37, D, BF, pad, offset) for _ in range(3))
    gain = randn(g, D)
    dx, dgain = ops.rmsnorm_backward(dy, h, gain, dres=dres)
    dx64, mag, dg64, dgmag = back64(dy, h, gain, 1e-6, dres)
    close(dx, dx64, BACK_U * mag + 2.0 ** -8 * dx64.abs(), "dx")
    close(dgain, dg64, (37 + 8) * U * dgmag + NORM_U * dgmag, "dgain")
    # in place of either input
    for k in (0, 1):
        a = [dy.clone(), dres.clone()]
        got, again = ops.rmsnorm_backward(a[0], h, gain, dres=a[1], out=a[k])
        assert got is a[k] and torch.equal(got, dx) and torch.equal(again, dgain)


def test_norm_backward_is_the_difference_quotient(ops):
    """<dx, d> and <dgain, e> against central differences of the forward
    formula in 64 bits: the step 1e-5 leaves a relative error of about 1e-9."""
    g = gen(11)
    T, D, eps = 6, 300, 1e-3
    h, dy, gain = randn(g, T, D), randn(g, T, D), 1 + 0.1 * randn(g, D)
    dx, dgain = ops.rmsnorm_backward(dy, h, gain, eps=eps)

    def f(h_, gain_):
        return (norm64(h_, gain_, None, eps)[1] * dy.double()).sum().item()

    for seed in range(4):
        d, e = randn(gen(seed), T, D).double(), randn(gen(seed + 9), D).double()
        h64, g64, s = h.double(), gain.double(), 1e-5
        want = (f(h64 + s * d, g64) - f(h64 - s * d, g64)) / (2 * s)
        assert abs((dx.double() * d).sum().item() - want) <= 1e-5 * (dx.double() * d).abs().sum().item()
        want = (f(h64, g64 + s * e) - f(h64, g64 - s * e)) / (2 * s)
        assert abs((dgain.double() * e).sum().item() - want) <= 1e-5 * (dgain.double() * e).abs().sum().item()


# ---- the product of 8-bit integers ----

def ints(g, R, K, ld=None, lo=-127, hi=127):
    return torch.randint(lo, hi + 1, (R, ld or K), generator=g, device="cuda", dtype=torch.int8)[:, :K]


def check_product(ops, xq, wq, g, dtype):
    T, V = xq.shape[0], wq.shape[0]
    xs = 0.5 + torch.rand(T, generator=g, device="cuda")
    ws = (0.5 + torch.rand(V, generator=g, device="cuda")) * 1e-3
    out = ops.matmul_quant(xq, xs, wq, ws, dtype=dtype)
    x64, w64 = xq.double(), wq.double()
    acc, mag = x64 @ w64.T, x64.abs() @ w64.abs().T
    scale = xs.double()[:, None] * ws.double()
    # integer sums below 2^24 are exact in fp32; larger ones lose at most two
    # ulps per step of 16 products (the tensor cores truncate)
    lost = torch.where(mag < 2 ** 24, 0.0, (xq.shape[1] / 16 + 2) * 2.0 ** -22 * mag)
    close(out, acc * scale, lost * scale + (4 * U + out_u(dtype)) * (acc * scale).abs(), "product")
    assert ops.device_status() == E.EMBER_OK


MM_SHAPES = [(1, 1, 1), (1, 5, 3), (1, 1000, 64), (1, 3001, 896), (1, 129, 8192), (2, 640, 768), (3, 257, 80),
             (4, 1000, 112), (7, 511, 1003), (8, 2000, 2048), (8, 100, 32768), (9, 300, 64), (16, 256, 128),
             (17, 255, 144), (31, 1030, 896), (49, 5000, 896), (64, 512, 1000), (65, 700, 200), (127, 129, 272),
             (128, 1280, 512), (200, 1000, 4096), (257, 515, 1008), (400, 900, 65), (1000, 2049, 320), (33, 40, 8192),
             (12, 70000, 96), (0, 64, 64), (6, 20000, 256), (3, 17000, 2064), (2, 30, 20000),
             (64, 4161, 7856), (10, 500, 4099), (190, 300, 2048), (129, 255, 32768), (500, 1100, 3000)]


@pytest.mark.parametrize("T,V,K", MM_SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_product(ops, T, V, K, dtype):
    g = gen(T + V + K)
    ld = (K + 15) // 16 * 16
    check_product(ops, ints(g, T, K, ld), ints(g, V, K, ld), g, dtype)


@pytest.mark.parametrize("T,V,K,ldx,ldw", [(1, 100, 70, 71, 73), (5, 333, 1003, 1003, 1003), (40, 200, 96, 97, 96),
                                           (40, 200, 96, 96, 101), (130, 70, 77, 80, 77), (6, 60, 64, 128, 192),
                                           (60, 600, 64, 128, 192)])
def test_product_of_strided_rows(ops, T, V, K, ldx, ldw):
    g = gen(K)
    check_product(ops, ints(g, T, K, ldx), ints(g, V, K, ldw), g, F32)


@pytest.mark.parametrize("T", [1, 40, 150])
def test_product_of_the_extremes(ops, T):
    """All 127, all -128 and alternating signs: the largest sums there are."""
    K, V = 4096, 300
    g = gen(3)
    x = torch.full((T, K), 127, device="cuda", dtype=torch.int8)
    w = torch.full((V, K), -128, device="cuda", dtype=torch.int8)
    w[1::3] = 127
    w[2::3, ::2] = 127
    check_product(ops, x, w, g, F32)
    x[:, ::2] = -128
    check_product(ops, x, w, g, F32)


@pytest.mark.parametrize("T", [1, 8, 30, 150])
def test_product_writes_its_rows_alone(ops, T):
    g = gen(8)
    K, V = 128, 301
    xq, wq = ints(g, T, K), ints(g, V, K)
    xs, ws = torch.ones(T, device="cuda"), torch.ones(V, device="cuda")
    b = torch.full((T + 2, V + 9), 7.0, device="cuda")
    ops.matmul_quant(xq, xs, wq, ws, dtype=F32, out=b[1:T + 1, 4:V + 4])
    assert torch.equal(b[1:T + 1, 4:V + 4].double(), xq.double() @ wq.double().T)
    assert (b[0] == 7).all() and (b[T + 1] == 7).all() and (b[:, :4] == 7).all() and (b[:, V + 4:] == 7).all()


@pytest.mark.parametrize("T", [2, 20])
def test_a_nan_scale_stays_in_its_row_or_column(ops, T):
    g = gen(9)
    xq, wq = ints(g, T, 64), ints(g, 70, 64)
    xs, ws = torch.ones(T, device="cuda"), torch.ones(70, device="cuda")
    xs[1], ws[3] = math.nan, math.inf
    out = ops.matmul_quant(xq, xs, wq, ws, dtype=F32)
    assert torch.isnan(out[1]).all() and not torch.isfinite(out[:, 3]).any()
    out[1], out[:, 3] = 0, 0
    assert torch.isfinite(out).all()


def test_the_8_bit_head_end_to_end(ops):
    """Hidden states and table in 8 bits against the product of what they stand for."""
    g = gen(4)
    T, V, D = 37, 1234, 768
    x, res, W = rows(g, T, D, BF), rows(g, T, D, BF), (randn(g, V, D) * 0.02).to(BF)
    wq, ws = ops.quantize_rows(W)
    q, scales, _ = ops.rmsnorm_quant(x, None, residual=res)
    out = ops.matmul_quant(q, scales, wq, ws, dtype=F32)
    y = ops.dequantize_rows(q, scales, dtype=F32).double()
    w = ops.dequantize_rows(wq, ws, dtype=F32).double()
    close(out, y @ w.T, 8 * U * (y.abs() @ w.abs().T), "logits")


# ---- the loss ----

def loss64(z, y, w, ignore, mean):
    z = z.double()
    T, V = z.shape
    valid = (y != ignore) & (y >= 0) & (y < V)
    n = int(valid.sum()) if mean else 1
    at = torch.where(valid, y, 0).long()[:, None]
    m = z.amax(1, keepdim=True)
    # from the maximum on: at the type's lowest value log V vanishes in z + log V even in 64 bits
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    nll = torch.where(valid, (torch.log(total) + (m - z.gather(1, at)))[:, 0], 0.0)
    g = torch.where(valid, torch.ones(T, device="cuda", dtype=torch.float64) if w is None else w.double(), 0.0)
    loss = torch.where(valid, g * nll, 0.0).sum() / max(n, 1)
    g = (g / max(n, 1))[:, None]
    p = e / total
    d = g * p
    d.scatter_add_(1, at, -g)
    # e^x for x = z - max: three roundings of x (the difference, the product
    # by log2 e, a rescaling by another maximum), each a relative u |x|, and a
    # few ulps of 2^x; the sum passes through V / 1024 + 60 additions
    far = (m - z).clamp(max=200.0)
    sums = (V / 1024 + 100) * U
    dbound = g.abs() * p * (6 * far * U + 32 * U + sums) + 4 * U * d.abs() + U * g.abs() * (p > 0.5)
    nbound = sums + 64 * U + 4 * U * (m.abs() + lse.abs() + z.gather(1, at).abs())[:, 0]
    return loss, nll, d, dbound, torch.where(valid, nbound, 0.0), g


def check_loss(ops, z, y, w=None, ignore=-100, mean=True, dtype=None, **kw):
    loss, nll, d = ops.softmax_loss(z, y, weights=w, ignore_index=ignore, reduction="mean" if mean else "sum",
                                    grad_dtype=dtype, **kw)
    l64, n64, d64, db, nb, g = loss64(z, y, w, ignore, mean)
    close(nll, n64, nb, "nll")
    close(d, d64, db + (out_u(d.dtype) + U) * d64.abs(), "dlogits")
    close(loss, l64, (g.abs()[:, 0] * nb).sum() + 8 * U * (g.abs()[:, 0] * n64.abs()).sum(), "loss")
    return loss, nll, d


LOSS_SHAPES = [(1, 1), (1, 2), (3, 7), (2, 8), (5, 65), (9, 1000), (4, 4096), (33, 5003), (7, 50257), (3, 128256),
               (200, 2048), (2, 262144), (1, 262161), (2, 300001), (170, 32768), (400, 777), (1, 16384)]


@pytest.mark.parametrize("T,V", LOSS_SHAPES)
@pytest.mark.parametrize("zt,dt", [(BF, BF), (F32, F32), (F32, BF), (BF, F32)])
def test_loss(ops, T, V, zt, dt):
    g = gen(T + V)
    z = rows(g, T, V, zt, scale=3.0)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    if T > 2:
        y[1] = -100
    check_loss(ops, z, y, dtype=dt)
    assert ops.device_status() == E.EMBER_OK


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (47, 5), (7, 8)])
@pytest.mark.parametrize("V", [5, 64, 1003, 50257])
@pytest.mark.parametrize("zt,dt", [(BF, BF), (F32, BF), (F32, F32)])
def test_loss_of_strided_rows(ops, V, pad, offset, zt, dt):
    g = gen(V + pad)
    T = 21
    z = rows(g, T, V, zt, pad, offset, scale=2.0)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    w = randn(g, T)
    check_loss(ops, z, y, w, mean=False, dtype=dt)
    guard = torch.full((T, V + 11), 7.0, device="cuda", dtype=dt)
    check_loss(ops, z, y, w, dtype=dt, out=guard[:, 3:V + 3])
    assert (guard[:, :3] == 7).all() and (guard[:, V + 3:] == 7).all()


@pytest.mark.parametrize("V", [100, 50257, 262145])
def test_loss_in_place_and_alone(ops, V):
    g = gen(V)
    z = rows(g, 19, V, BF, scale=2.0)
    y = torch.randint(0, V, (19,), generator=g, device="cuda")
    loss, nll, d = ops.softmax_loss(z, y)
    l2, n2, none = ops.softmax_loss(z, y, grad=False)
    assert none is None and torch.equal(nll, n2) and torch.equal(loss, l2)
    z2 = z.clone()
    l3, n3, d3 = ops.softmax_loss(z2, y, out=z2)
    assert d3 is z2 and torch.equal(d3, d) and torch.equal(n3, nll) and torch.equal(l3, loss)


@pytest.mark.parametrize("V", [40, 1003, 50257, 300000])
def test_masks_and_lowest_values(ops, V):
    g = gen(V)
    z = rows(g, 8, V, F32)
    y = torch.randint(0, V // 2, (8,), generator=g, device="cuda")
    z[0, V // 2:] = -math.inf
    z[1, V // 2:] = torch.finfo(F32).min
    z[2] = torch.finfo(F32).min  # a row of lowest values is uniform
    z[3] = torch.finfo(BF).min
    z[4, :] = -math.inf
    z[4, y[4]] = 1.5  # nothing but the target
    z[5] *= 1e4
    z[6] += 1e6
    check_loss(ops, z, y)


@pytest.mark.parametrize("V", [40, 1003, 50257, 300000])
def test_rows_without_a_distribution(ops, V):
    g = gen(V)
    z = rows(g, 6, V, F32)
    y = torch.randint(0, V, (6,), generator=g, device="cuda")
    z[1] = -math.inf
    z[2, 3] = math.nan
    z[3, 4] = math.inf
    z[4, y[4]] = -math.inf  # the target masked out: an infinite loss, a finite gradient
    loss, nll, d = ops.softmax_loss(z, y, reduction="sum")
    assert nll[1] == math.inf and (d[1] == 0).all()
    assert torch.isnan(nll[2:4]).all() and torch.isnan(d[2:4]).all() and torch.isnan(loss)
    assert nll[4] == math.inf
    p = torch.softmax(z[4].double(), 0)
    p[y[4]] = -1
    assert torch.allclose(d[4].double(), p, rtol=1e-4, atol=1e-12)
    for k in (0, 5):
        assert torch.isfinite(nll[k]) and torch.isfinite(d[k]).all()


@pytest.mark.parametrize("V", [64, 50257, 270001])
def test_targets_that_do_not_count(ops, V):
    g = gen(V)
    z = rows(g, 7, V, BF)
    z[2] = math.nan  # an ignored row is not looked at
    y = torch.randint(0, V, (7,), generator=g, device="cuda")
    y[2] = y[5] = 3
    w = randn(g, 7)
    w[5] = math.nan
    loss, nll, d = ops.softmax_loss(z, y, weights=w, ignore_index=3)
    assert (nll[[2, 5]] == 0).all() and (d[[2, 5]] == 0).all() and torch.isfinite(loss) and torch.isfinite(d).all()
    assert ops.device_status() == E.EMBER_OK
    y[0], y[1] = V, -1
    loss, nll, d = ops.softmax_loss(z, y, weights=w, ignore_index=3)
    assert (nll[:2] == 0).all() and (d[:2] == 0).all()
    assert ops.device_status() == E.EMBER_ERR_ID_OUT_OF_RANGE
    assert ops.device_status() == E.EMBER_OK
    y[:] = 3
    loss, nll, d = ops.softmax_loss(z, y, ignore_index=3)
    assert loss == 0 and (nll == 0).all() and (d == 0).all()
    loss, nll, d = ops.softmax_loss(z[:0], y[:0])
    assert loss == 0 and nll.shape == (0,) and d.shape == (0, V)


def test_loss_gradient_is_the_difference_quotient(ops):
    g = gen(2)
    T, V = 5, 400
    z, y, w = randn(g, T, V), torch.randint(0, V, (T,), generator=g, device="cuda"), randn(g, T)
    d = ops.softmax_loss(z, y, weights=w)[2].double()
    for seed in range(4):
        e, s = randn(gen(seed), T, V).double(), 1e-5
        want = (loss64(z.double() + s * e, y, w, -100, True)[0] - loss64(z.double() - s * e, y, w, -100, True)[0]) / (2 * s)
        assert abs((d * e).sum() - want) <= 1e-5 * (d * e).abs().sum()


# ---- norm and clipping of gradients ----

def check_clip(ops, grads, max_norm, in_place=False):
    n64 = math.sqrt(sum(t.double().square().sum().item() for t in grads))
    # up to 8 squares in a chain of fp32, two joins, then 64 bits; the root
    # halves it and rounds
    assert abs(ops.grad_norm(grads).item() - n64) <= 8 * U * n64 + TINY
    src = [t.clone() for t in grads]
    out = src if in_place else [torch.empty_like(t) for t in grads]
    norm = ops.clip_grads(src, max_norm, out=None if in_place else out)
    assert abs(norm.item() - n64) <= 8 * U * n64 + TINY
    c = min(1.0, max_norm / (n64 + 1e-6))
    for o, t in zip(out, grads):
        want = t.double() * c
        close(o, want, (16 * U + out_u(t.dtype)) * want.abs() + out_u(t.dtype) * TINY, "clipped")
    return norm


SETS = [[1], [7], [0, 5, 0], [4096], [4097, 3], [100000, 1, 33], [3000000, 17], [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 17],
        [20000000, 5000001, 64]]


@pytest.mark.parametrize("sizes", SETS, ids=str)
@pytest.mark.parametrize("types", [(F32,), (BF,), (F32, BF)])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(ops, sizes, types, in_place):
    g = gen(sum(sizes))
    grads = [(randn(g, n) * 10.0 ** (k % 4 - 2)).to(types[k % len(types)]) for k, n in enumerate(sizes)]
    norm = math.sqrt(sum(t.double().square().sum().item() for t in grads))
    check_clip(ops, grads, 0.3 * norm, in_place)
    check_clip(ops, grads, 2.0 * norm, in_place)
    check_clip(ops, grads, 0.0, in_place)


def test_clip_of_many_tensors(ops):
    g = gen(1)
    grads = [randn(g, 1 + (37 * k) % 301).to(BF if k % 3 == 0 else F32) for k in range(2500)]
    check_clip(ops, grads, 1.0)
    check_clip(ops, grads[:65], 1.0, in_place=True)


@pytest.mark.parametrize("t", [BF, F32])
def test_clip_off_the_boundaries(ops, t):
    """Views of one buffer at odd places, into another's at other odd places."""
    g = gen(6)
    b = randn(g, 200000).to(t)
    cuts = [0, 1, 4, 9, 1000, 1003, 50001, 120000, 199993]
    grads = [b[i:j] for i, j in zip(cuts, cuts[1:])]
    check_clip(ops, grads, 1.0)
    o = torch.full((200010,), 7.0, device="cuda", dtype=t)
    outs = [o[i + 5:j + 5] for i, j in zip(cuts, cuts[1:])]
    ops.clip_grads(grads, 1.0, out=outs)
    n64 = b[:199993].double().norm().item()
    want = b[:199993].double() / (n64 + 1e-6)
    close(o[5:199998], want, (16 * U + out_u(t)) * want.abs(), "clipped")
    assert (o[:5] == 7).all() and (o[199998:] == 7).all()


@pytest.mark.parametrize("scale", [1e-38, 1e-25, 1e-14, 1e15, 1e18, 3e37])
def test_norm_does_not_leave_the_range(ops, scale):
    grads = [randn(gen(3), 70000).clamp(-3, 3) * scale, torch.zeros(50000, device="cuda")]
    n64 = grads[0].double().norm().item()
    norm = ops.grad_norm(grads).item()
    if n64 < 3.4e38:
        assert abs(norm - n64) <= 8 * U * n64
    else:
        assert norm == math.inf


def test_clip_of_infinite_and_nan_gradients(ops):
    a, b = torch.ones(1000, device="cuda"), torch.ones(70, device="cuda")
    a[3] = math.inf
    out = [torch.empty_like(t) for t in (a, b)]
    assert ops.clip_grads([a, b], 1.0, out=out) == math.inf
    assert torch.isnan(out[0][3]) and (out[1] == 0).all() and (out[0][:3] == 0).all()
    b[1] = math.nan
    assert torch.isnan(ops.clip_grads([a, b], 1.0, out=out))
    assert torch.isnan(out[0]).all() and torch.isnan(out[1]).all()


def test_no_gradients(ops):
    assert ops.grad_norm([]) == 0 and ops.clip_grads([], 1.0) == 0
    assert ops.clip_grads([torch.empty(0, device="cuda")], 1.0) == 0


# ---- streams, repetition ----

def test_the_same_bits_on_every_run_and_on_another_stream(ops):
    g = gen(7)
    x, res, gain = rows(g, 500, 1024, BF), rows(g, 500, 1024, F32), randn(g, 1024)
    z, y = rows(g, 50, 50257, F32), torch.randint(0, 50257, (50,), generator=g, device="cuda")
    grads = [randn(g, 100000), randn(g, 77)]
    xq, wq = ints(g, 60, 512), ints(g, 3000, 512)
    xs, ws = torch.rand(60, generator=g, device="cuda"), torch.rand(3000, generator=g, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    own = Ops()

    def all_of(o, stream):
        out = [*o.rmsnorm(x, gain, residual=res, stream=stream), *o.rmsnorm_quant(x, gain, stream=stream)[:2],
               *o.rmsnorm_backward(x, x, gain, stream=stream), *o.softmax_loss(z, y, stream=stream),
               o.matmul_quant(xq, xs, wq, ws, stream=stream), o.matmul_quant(xq[:3], xs[:3], wq, ws, stream=stream)]
        buf = [torch.empty_like(t) for t in grads]
        out += [o.clip_grads(grads, 1.0, out=buf, stream=stream), *buf]
        torch.cuda.synchronize()
        return out

    first = all_of(ops, None)
    for o, s in ((ops, None), (own, side), (own, side.cuda_stream)):
        for a, b in zip(first, all_of(o, s)):
            assert torch.equal(a, b)


def test_calls_follow_the_work_before_them(ops):
    """Inputs written on the stream right before each call, many times: no
    kernel may start reading before they are there."""
    g = gen(8)
    x = rows(g, 64, 512, F32)
    base = x.clone()
    z = rows(g, 16, 1000, F32)
    zb, y = z.clone(), torch.randint(0, 1000, (16,), generator=g, device="cuda")
    big = torch.zeros(1 << 26, device="cuda")
    for k in range(1, 20):
        big.add_(1.0)
        x.copy_(base * k)
        z.copy_(zb / k)
        out, _ = ops.rmsnorm(x, None)
        loss, nll, d = ops.softmax_loss(z, y)
        norm = ops.grad_norm([out, d])
        torch.cuda.synchronize()
        assert torch.equal(out, ops.rmsnorm(base * k, None)[0])
        l2, _, d2 = ops.softmax_loss(zb / k, y)
        assert torch.equal(l2, loss) and torch.equal(d2, d)
        assert norm == ops.grad_norm([out, d2])


def test_graph_capture(ops):
    g = gen(9)
    x, z = rows(g, 8, 256, BF), rows(g, 8, 1000, BF)
    y = torch.randint(0, 1000, (8,), generator=g, device="cuda")
    xq, wq = ints(g, 20, 128), ints(g, 500, 128)
    xs, ws = torch.rand(20, generator=g, device="cuda"), torch.rand(500, generator=g, device="cuda")
    own = Ops()
    grads = [randn(g, 1000)]
    buf = [torch.empty_like(grads[0])]

    def body():
        own.clip_grads(grads, 1.0, out=buf)
        return [own.rmsnorm(x, None)[0], own.softmax_loss(z, y)[2], own.matmul_quant(xq, xs, wq, ws),
                own.rmsnorm_backward(x, x, None)[0]]

    want = [t.clone() for t in body()] + [buf[0].clone()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = body()
    buf[0].zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got + buf, want):
        assert torch.equal(a, b)


# ---- past 2^31 elements ----

def test_offsets_past_32_bits(ops):
    """The last rows of matrices of more than 2^31 elements, against calls on
    those rows alone."""
    g = gen(10)
    T, D = 70000, 32768
    x = torch.empty(T, D, device="cuda", dtype=BF)
    x[:8] = rows(g, 8, D, BF)
    x[8:-8] = 1.0
    x[-8:] = rows(g, 8, D, BF)
    y, h = ops.rmsnorm(x, None, residual=x)
    y2, h2 = ops.rmsnorm(x[-8:].clone(), None, residual=x[-8:].clone())
    assert torch.equal(y[-8:], y2) and torch.equal(h[-8:], h2)
    del h
    q, s = ops.quantize_rows(x)
    q2, s2 = ops.quantize_rows(x[-8:].clone())
    assert torch.equal(q[-8:], q2) and torch.equal(s[-8:], s2)
    assert torch.equal(ops.dequantize_rows(q, s, out=y)[-8:], ops.dequantize_rows(q2, s2))
    del q
    dx, _ = ops.rmsnorm_backward(x, x, None, out=y)
    assert torch.equal(dx[-8:], ops.rmsnorm_backward(x[-8:].clone(), x[-8:].clone(), None)[0])
    del dx, y
    z = x.view(-1)[:17000 * 128256].view(17000, 128256)
    z[-3:] = rows(g, 3, 128256, BF)
    t = torch.randint(0, 128256, (17000,), generator=g, device="cuda")
    _, nll, d = ops.softmax_loss(z, t, reduction="sum")
    _, nll2, d2 = ops.softmax_loss(z[-3:].clone(), t[-3:], reduction="sum")
    assert torch.equal(nll[-3:], nll2) and torch.equal(d[-3:], d2)
    out = [d.view(-1)]
    norm = ops.clip_grads([z.view(-1)], 1.0, out=out)
    want = z[-1].double() / (norm.item() + 1e-6)
    close(d[-1], want, 2.0 ** -8 * want.abs() + 1e-6 * want.abs(), "clipped")
    assert norm.item() == ops.grad_norm([z.view(-1)]).item()


@pytest.mark.parametrize("T", [2, 40])
def test_tables_and_logits_past_32_bits(ops, T):
    g = gen(11)
    V, K = 140000, 16384  # 2.3e9 bytes of table
    wq = torch.ones(V, K, device="cuda", dtype=torch.int8)
    wq[-300:] = ints(g, 300, K)
    xq = ints(g, T, K)
    xs, ws = torch.rand(T, generator=g, device="cuda"), torch.rand(V, generator=g, device="cuda")
    out = ops.matmul_quant(xq, xs, wq, ws, dtype=F32)
    assert torch.equal(out[:, -256:], ops.matmul_quant(xq, xs, wq[-256:].clone(), ws[-256:].clone(), dtype=F32))
    del wq, out
    T, V, K = 18000, 128000, 64
    wq, xq = ints(g, V, K), ints(g, T, K)
    xs, ws = torch.rand(T, generator=g, device="cuda"), torch.rand(V, generator=g, device="cuda")
    out = ops.matmul_quant(xq, xs, wq, ws)
    assert torch.equal(out[-200:], ops.matmul_quant(xq[-200:], xs[-200:], wq, ws))
    assert ops.device_status() == E.EMBER_OK


# ---- waits that run out ----

@pytest.mark.parametrize("T,V,K", [(40, 3000, 8192), (300, 9000, 2048)])
def test_a_wait_that_gives_up_is_reported(cuda_device, T, V, K):
    """With a limit of 1 ns the waits for the first copies run out: the calls
    return, the status says so, and the next calls are right."""
    ops, g = Ops(cuda_device), gen(12)
    xq, wq = ints(g, T, K), ints(g, V, K)
    xs, ws = torch.rand(T, generator=g, device="cuda"), torch.rand(V, generator=g, device="cuda")
    z, y = rows(g, T, 100000, BF), torch.randint(0, 100000, (T,), generator=g, device="cuda")
    want = ops.matmul_quant(xq, xs, wq, ws)
    wanted = ops.softmax_loss(z, y)
    try:
        ops.set_wait_limit_ns(1)
        ops.matmul_quant(xq, xs, wq, ws)
        assert ops.device_status() == E.EMBER_ERR_TIMEOUT
        assert ops.device_status() == E.EMBER_OK
        ops.softmax_loss(z, y)
        assert ops.device_status() in (E.EMBER_OK, E.EMBER_ERR_TIMEOUT)  # a copy may land before the clock is read
    finally:
        ops.set_wait_limit_ns(0)
    for _ in range(2):
        assert torch.equal(ops.matmul_quant(xq, xs, wq, ws), want)
        for a, b in zip(ops.softmax_loss(z, y), wanted):
            assert torch.equal(a, b)
        assert ops.device_status() == E.EMBER_OK


class _Passes:
    """A binding that takes no call."""

    def __getattr__(self, name):
        return lambda *a: None


class _Counts:
    """The binding, with the names of the calls it took."""

    def __init__(self, binding):
        self.binding, self.took = binding, []

    def __getattr__(self, name):
        f = getattr(self.binding, name)

        def call(*a):
            r = f(*a)
            if r is not None:
                self.took.append(name)
            return r
        return call


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [96, 1003])
def test_compiled_calls_give_what_the_others_give(dtype, D):
    """Every operator through the compiled call and through the module's own
    marshalling: equal bits, shapes, strides and types."""
    from paper_2607_01455_gb300 import Ops
    g = torch.Generator(device="cuda")
    g.manual_seed(D)

    def new(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    T, V = 37, 517
    x, res, dy, gain = new(T, D), new(T, D), new(T, D), new(D)
    z, w = new(T, V), torch.rand(T, generator=g, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    padded = torch.zeros(T, V + 11, device="cuda", dtype=dtype)[:, :V].copy_(z)
    grads = [new(n) for n in (1, 7, 4096, 0, 33)]
    W = new(V, D)

    def run(o):
        wq, ws = o.quantize_rows(W)
        xq, xs, _ = o.rmsnorm_quant(x, gain)
        outs = [torch.empty_like(t) for t in grads]
        results = [
            *o.rmsnorm(x, gain, residual=res), *o.rmsnorm(x, None), *o.rmsnorm_quant(x, gain, residual=res),
            *o.rmsnorm_backward(dy, x, gain), *o.rmsnorm_backward(dy, x, None, dres=res, out=torch.empty_like(x)),
            o.dequantize_rows(xq, xs, dtype), o.matmul_quant(xq, xs, wq, ws, dtype),
            *o.softmax_loss(z, y), *o.softmax_loss(padded, y, weights=w, reduction="sum", grad_dtype=torch.float32),
            *o.softmax_loss(z, y.int(), grad=False), o.grad_norm(grads), o.clip_grads(grads, 0.5, out=outs), *outs]
        assert o.device_status() == 0
        return results

    a, b = Ops(), Ops()
    a._fast, b._fast = _Counts(a._fast), _Passes()
    run(a)  # the workspace grows on the way
    a._fast.took.clear()
    for p, q in zip(run(a), run(b), strict=True):
        assert (p is None) == (q is None)
        if p is not None:
            assert p.shape == q.shape and p.stride() == q.stride() and p.dtype == q.dtype and torch.equal(p, q)
    assert a._fast.took == ["rmsnorm_quant", "rmsnorm", "rmsnorm", "rmsnorm_quant", "rmsnorm_backward",
                            "rmsnorm_backward", "dequantize_rows", "matmul_quant", "softmax_loss", "softmax_loss",
                            "softmax_loss", "grad_norm", "clip_grads"]


@pytest.mark.gpu
def test_compiled_calls_keep_no_references():
    import sys

    from paper_2607_01455_gb300 import Ops
    o = Ops()
    x, out, gain = torch.randn(5, 64, device="cuda"), torch.empty(5, 64, device="cuda"), torch.ones(64, device="cuda")
    grads = [torch.randn(9, device="cuda") for _ in range(3)]
    y = torch.zeros(5, dtype=torch.int64, device="cuda")
    held = [x, out, gain, grads, grads[0], y]

    def calls():
        o.rmsnorm(x, gain, out=out)
        o.rmsnorm(x, gain, residual=x, residual_out=out)
        o.rmsnorm_quant(x, gain)
        o.rmsnorm_backward(x, x, gain, out=out)
        o.softmax_loss(x, y, out=out)
        o.clip_grads(grads, 1.0)
        with pytest.raises(Exception):
            o.rmsnorm(x, gain, out=out[:4])

    calls()
    before = [sys.getrefcount(t) for t in held]
    torch.cuda.synchronize()
    memory = torch.cuda.memory_allocated()
    for _ in range(8):
        calls()
    torch.cuda.synchronize()
    assert [sys.getrefcount(t) for t in held] == before and torch.cuda.memory_allocated() == memory


@pytest.mark.gpu
def test_clipping_refuses_a_limit_that_is_no_number():
    import ctypes

    from paper_2607_01455_gb300 import Ops
    o = Ops()
    grads = [torch.ones(4, device="cuda")]
    o.clip_grads(grads, 8.0)
    for bad in (None, "1"):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            o.clip_grads(grads, bad)
    assert torch.equal(grads[0], torch.ones(4, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", [(384, 300), (385, 300), (513, 5003), (1024, 8000), (1025, 8000), (1100, 1000), (5000, 129)])
@pytest.mark.parametrize("zt", [BF, F32])
def test_loss_with_and_without_launches_of_its_own_for_the_count(ops, T, V, zt):
    """Numbers of tokens around the limits up to which one launch does it all;
    weights of tokens that do not count reach nothing, not as NaN either."""
    g = gen(T + V)
    z = rows(g, T, V, zt, scale=3.0)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    w = randn(g, T)
    ignored = torch.arange(T, device="cuda") % 7 == 3
    y[ignored] = -100
    check_loss(ops, z, y)
    w64 = torch.where(ignored, 0.0, w)
    w[ignored] = float("nan")
    got = ops.softmax_loss(z, y, weights=w)
    want = check_loss(ops, z, y, w64)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert ops.device_status() == E.EMBER_OK
    y[5] = V
    loss, nll, d = ops.softmax_loss(z, y)
    y[5] = -100
    assert torch.equal(loss, ops.softmax_loss(z, y)[0]) and nll[5] == 0 and (d[5] == 0).all()
    assert ops.device_status() == E.EMBER_ERR_ID_OUT_OF_RANGE


@pytest.mark.gpu
@pytest.mark.parametrize("n", [63, 64, 65, 256, 257, 1024, 1025])
def test_clip_around_the_launches_limits(ops, n):
    """Numbers of tensors at which the next longer list, or another launch, begins."""
    g = gen(n)
    grads = [randn(g, 1 + (53 * k) % 211).to(BF if k % 4 == 1 else F32) for k in range(n)]
    check_clip(ops, grads, 0.7)
    check_clip(ops, grads[:-1] + [randn(g, 6000000)], 0.7, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,K", [(9, 1000, 64), (16, 4863, 2048), (24, 1000, 512), (76, 1000, 272), (72, 1024, 1003),
                                   (73, 1056, 2048), (7, 16385, 1008), (8, 16384, 100), (300, 33, 640), (304, 8, 16)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_product_of_token_groups(ops, T, V, K, dtype):
    """More than eight tokens by a small table, around the limits of the form that takes them in groups."""
    g = gen(T + V + K)
    ld = (K + 15) // 16 * 16
    x, w = ints(g, T, K, ld), ints(g, V, K, ld)
    check_product(ops, x, w, g, dtype)
    xs, ws = torch.rand(T, generator=g, device="cuda"), torch.rand(V, generator=g, device="cuda")
    guard = torch.full((T + 3, V + 5), 7.0, device="cuda", dtype=dtype)
    out = ops.matmul_quant(x, xs, w, ws, dtype=dtype, out=guard[1:T + 1, 2:V + 2])
    assert torch.equal(out, ops.matmul_quant(x, xs, w, ws, dtype=dtype))
    guard[1:T + 1, 2:V + 2] = 7
    assert (guard == 7).all()
