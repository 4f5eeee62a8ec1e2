"""The operators where their kernels' forms differ: codes next to a tie, rows
masked far below zero, and the forms that only longer calls take.  References and
bounds as in test_ops_gpu.
"""
import math

import pytest
import torch
from test_ops_gpu import (BACK_U, BF, F32, NORM_U, U, back64, check_loss, check_rows8, close, gen, norm64, out_u, randn,
                          rows)

from paper_2607_01455_gb300 import Ops
from paper_2607_01455_gb300 import ember as E

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops(cuda_device):
    return Ops(cuda_device)


# ---- 8-bit codes: the fp32 quotient y / scale, rounded to nearest even ----

def over_127(x):
    """x / 127, rounded once (by a Python number torch multiplies by its reciprocal)."""
    return x / torch.full_like(x, 127.0)


def near_ties(g, D):
    """D values of a row, the largest in front: the others lie within two
    steps of fp32 around (m + 1/2) scale."""
    top = (1.0 + torch.rand(1, generator=g, device="cuda")).float()
    scale = top / 127
    m = torch.randint(-126, 126, (D - 1,), generator=g, device="cuda")
    y = ((m + 0.5).double() * scale.double()).float()
    by = torch.randint(-2, 3, (D - 1,), generator=g, device="cuda")
    for step in (1, 2):
        y = torch.where(by >= step, torch.nextafter(y, y + 1), y)
        y = torch.where(by <= -step, torch.nextafter(y, y - 1), y)
    return torch.cat([top, y])


@pytest.mark.parametrize("T,D,pad", [(3, 1003, 0), (1, 4096, 0), (400, 512, 0), (200, 1003, 0), (40, 8200, 0),
                                     (5, 8193, 0), (33, 96, 5)])
def test_codes_next_to_a_tie(ops, T, D, pad):
    g = gen(T + D)
    x = torch.zeros(T, D + pad, device="cuda")[:, :D]
    for t in range(T):
        x[t] = near_ties(g, D) * 2.0 ** (t % 40 - 20)
    q, scales = ops.quantize_rows(x)
    assert torch.equal(scales, over_127(x.abs().amax(1)))
    assert torch.equal(q, torch.round(x / scales[:, None]).to(torch.int8))


@pytest.mark.parametrize("t", [BF, F32])
def test_codes_of_a_table(ops, t):
    x = (randn(gen(1), 5000, 4096) * 0.02).to(t)
    q, scales = ops.quantize_rows(x)
    assert torch.equal(q, torch.round(x.float() / scales[:, None]).to(torch.int8))


@pytest.mark.parametrize("T,D", [(2, 256), (3, 1024), (300, 4096), (2500, 4096), (9, 16384)])
@pytest.mark.parametrize("offset", [0, 1])
def test_codes_of_the_norm_next_to_a_tie(ops, T, D, offset):
    """Rows of ones of either sign: with eps = 0 the norm is exactly 1 and y the gain with their signs."""
    g = gen(D)
    gain = near_ties(g, D)
    x = torch.randint(0, 2, (T, D + offset), generator=g, device="cuda").float()[:, offset:] * 2 - 1
    q, scales, _ = ops.rmsnorm_quant(x, gain, eps=0.0)
    assert torch.equal(scales, over_127(gain[:1]).expand(T))
    assert torch.equal(q, torch.round(x * gain / scales[:, None]).to(torch.int8))


# ---- masked entries of rows far below zero ----

def below(g, T, V, t, base, pad=0, offset=0):
    z = rows(g, T, V, t, pad, offset)
    z += base
    z[:, V // 2:] = -math.inf
    z[1::3, :V // 4] = -math.inf
    return z, torch.randint(V // 4, V // 2, (T,), generator=g, device="cuda")


@pytest.mark.parametrize("T,V", [(6, 40), (6, 1003), (8, 50257), (4, 262144), (3, 300000), (1030, 1003), (1100, 5003),
                                 (1030, 30000), (1030, 50257), (3, 600001)])
@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("base", [-100.0, -1e4, -1e30])
def test_masks_of_rows_far_below_zero(ops, T, V, t, base):
    """Where all that a thread holds of a row is masked out, the row's maximum
    may still be any number: the masked gradients are zero, the others those of the row."""
    z, y = below(gen(V), T, V, t, base)
    for w in (None, torch.full((T,), 1e6, device="cuda")):
        loss, nll, d = check_loss(ops, z, y, w)
        assert (d[:, V // 2:] == 0).all() and (d[1::3, :V // 4] == 0).all()
    assert ops.device_status() == E.EMBER_OK


@pytest.mark.parametrize("V", [40, 50257])
def test_a_nan_beside_masks_far_below_zero(ops, V):
    """A NaN still reaches the whole of its row, whichever thread sees it, and no other row."""
    z, y = below(gen(V), 5, V, F32, -200.0)
    z[0, V - 1] = z[1, V // 4] = z[2, 0] = math.nan
    loss, nll, d = ops.softmax_loss(z, y)
    assert torch.isnan(nll[:3]).all() and torch.isnan(d[:3]).all() and torch.isnan(loss)
    assert torch.isfinite(nll[3:]).all() and torch.isfinite(d[3:]).all()


# ---- waits of the loss that run out ----

@pytest.mark.parametrize("T,V", [(60, 500000), (1100, 500000), (1100, 60000), (40, 20000)])
@pytest.mark.parametrize("ignored", [0, 2])
def test_a_wait_of_the_loss_that_gives_up_is_reported(cuda_device, T, V, ignored):
    """Rows of two and more CTAs: with a limit of 1 ns the wait for the first
    copy gives up or, where there is none to wait for, that for the other CTAs'
    sums, which have only just been sent.  Each call returns, the status says so,
    and later calls give the bits that earlier ones gave."""
    ops, g = Ops(cuda_device), gen(13)
    z, y = rows(g, T, V, BF), torch.randint(0, V, (T,), generator=g, device="cuda")
    if ignored:
        y[::ignored] = -100
    want = [t.clone() for t in ops.softmax_loss(z, y)]
    assert ops.device_status() == E.EMBER_OK
    try:
        ops.set_wait_limit_ns(1)
        for _ in range(10):
            ops.softmax_loss(z, y)
            assert ops.device_status() == E.EMBER_ERR_TIMEOUT
            assert ops.device_status() == E.EMBER_OK  # cleared by the reading
    finally:
        ops.set_wait_limit_ns(0)
    for _ in range(2):
        for a, b in zip(ops.softmax_loss(z, y), want):
            assert torch.equal(a, b)
        assert ops.device_status() == E.EMBER_OK


# ---- streams by their handle ----

def test_streams_by_their_handle(ops):
    """The handle 0 is the default stream, any other the stream that has it."""
    side = torch.cuda.Stream()
    for on in (None, side):
        with torch.cuda.stream(on):
            for s in (torch.cuda.default_stream(), side):
                with ops._on(s.cuda_stream):
                    assert torch.cuda.current_stream().cuda_stream == s.cuda_stream


def test_calls_on_the_handle_0_follow_the_default_stream(ops):
    """Inputs written by long work on the default stream right before each call."""
    x = torch.zeros(300, 1024, device="cuda")
    big = torch.zeros(1 << 28, device="cuda")
    ops.rmsnorm(x, None)
    for k in range(1, 6):
        big.add_(1.0)
        x.fill_(float(k))
        y, _ = ops.rmsnorm(x, None, eps=0.0, stream=0)
        torch.cuda.synchronize()
        assert (y == 1).all()
        x.zero_()


# ---- forms that longer calls take ----

TYPES = [(BF, None), (BF, BF), (BF, F32), (F32, None), (F32, BF), (F32, F32)]


@pytest.mark.parametrize("T,D", [(2500, 1032), (1000, 4104), (700, 8192), (4400, 8192), (400, 8200),
                                 (320, 12800), (310, 16384)])
@pytest.mark.parametrize("xt,rt", TYPES)
def test_long_calls_of_the_norm(ops, T, D, xt, rt):
    """Rows of whole groups, each CTA taking several of them, with and without 8 bits."""
    g = gen(T + D)
    x = rows(g, T, D, xt)
    res = None if rt is None else rows(g, T, D, rt, scale=2.0)
    gain = 1 + 0.1 * randn(g, D)
    s64, y64 = norm64(x, gain, res, 1e-6)
    q, scales, h = ops.rmsnorm_quant(x, gain, residual=res)
    check_rows8(q, scales, y64, NORM_U)
    y, h2 = ops.rmsnorm(x, gain, residual=res)
    close(y, y64, (NORM_U + out_u(xt)) * y64.abs(), "y")
    if res is not None:
        close(h, s64, (U + out_u(rt)) * s64.abs(), "h")
        assert torch.equal(h, h2)
    for a, b in zip(ops.rmsnorm_quant(x, gain, residual=res), (q, scales, h)):
        assert (a is None and b is None) or torch.equal(a, b)
    # in place
    x2, r2 = x.clone(), None if res is None else res.clone()
    ops.rmsnorm(x2, gain, residual=r2, out=x2, residual_out=r2)
    assert torch.equal(x2, y) and (res is None or torch.equal(r2, h2))


@pytest.mark.parametrize("T,D", [(15000, 33), (12000, 130), (5000, 1003), (2000, 4095), (400, 8191)])
@pytest.mark.parametrize("xt,rt", TYPES)
def test_long_calls_of_odd_rows(ops, T, D, xt, rt):
    """Rows off the 16-byte boundaries, each CTA taking several of them."""
    g = gen(T + D)
    x = rows(g, T, D, xt)
    res = None if rt is None else rows(g, T, D, rt, scale=2.0)
    gain = 1 + 0.1 * randn(g, D)
    s64, y64 = norm64(x, gain, res, 1e-6)
    y, h = ops.rmsnorm(x, gain, residual=res)
    close(y, y64, (NORM_U + out_u(xt)) * y64.abs(), "y")
    q, scales, h2 = ops.rmsnorm_quant(x, gain, residual=res)
    check_rows8(q, scales, y64, NORM_U)
    if res is not None:
        close(h, s64, (U + out_u(rt)) * s64.abs(), "h")
        assert torch.equal(h, h2)
    else:
        q, scales = ops.quantize_rows(x)
        assert torch.equal(q, torch.round(x.float() / scales[:, None]).to(torch.int8))
    # rows at other places of the buffers, and in place
    guard = torch.full((T, D + 3), 7.0, device="cuda", dtype=xt)
    ops.rmsnorm(x, gain, residual=res, out=guard[:, 2:D + 2])
    assert torch.equal(guard[:, 2:D + 2], y) and (guard[:, :2] == 7).all() and (guard[:, D + 2:] == 7).all()
    x2, r2 = x.clone(), None if res is None else res.clone()
    ops.rmsnorm(x2, gain, residual=r2, out=x2, residual_out=r2)
    assert torch.equal(x2, y) and (res is None or torch.equal(r2, h))


@pytest.mark.parametrize("T,D", [(2000, 256), (1500, 1024), (1000, 4104), (700, 8192), (400, 8200), (320, 10000),
                                 (310, 16384), (200, 20000), (15000, 33), (5000, 1003), (2000, 4095), (400, 8191), (300, 9001),
                                 (200, 16401)])
@pytest.mark.parametrize("t,with_dres", [(BF, True), (BF, False), (F32, True), (F32, False)])
def test_long_calls_of_the_norm_backward(ops, T, D, t, with_dres):
    g = gen(T + D)
    h, dy = rows(g, T, D, t, scale=2.0), rows(g, T, D, t, scale=1e-3)
    dres = rows(g, T, D, t, scale=1e-3) if with_dres else None
    gain = 1 + 0.1 * randn(g, D)
    dx, dgain = ops.rmsnorm_backward(dy, h, gain, dres=dres)
    dx64, mag, dg64, dgmag = back64(dy, h, gain, 1e-6, dres)
    close(dx, dx64, BACK_U * mag + out_u(t) * dx64.abs(), "dx")
    close(dgain, dg64, (T + 8) * U * dgmag + NORM_U * dgmag, "dgain")
    d2 = dy.clone()
    again = ops.rmsnorm_backward(d2, h, gain, dres=dres, out=d2)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain)


@pytest.mark.parametrize("T,V", [(1500, 777), (1100, 30000), (1100, 50257), (1030, 64000), (1030, 128256), (1030, 270000)])
@pytest.mark.parametrize("zt,dt", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
def test_long_calls_of_the_loss(ops, T, V, zt, dt):
    """More tokens than one launch takes, by rows of each number of threads and CTAs."""
    g = gen(T + V)
    z = rows(g, T, V, zt, scale=3.0)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[5::11] = -100
    w = randn(g, T)
    loss, nll, d = check_loss(ops, z, y, w, dtype=dt)
    assert (nll[5::11] == 0).all() and (d[5::11] == 0).all()
    l2, n2, none = ops.softmax_loss(z, y, weights=w, grad=False)
    assert none is None and torch.equal(l2, loss) and torch.equal(n2, nll)
    if zt == dt:
        z2 = z.clone()
        l2, n2, d2 = ops.softmax_loss(z2, y, weights=w, out=z2)
        assert torch.equal(l2, loss) and torch.equal(n2, nll) and torch.equal(d2, d)
    assert ops.device_status() == E.EMBER_OK
