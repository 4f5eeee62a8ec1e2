"""The 4-bit table's operators and sampling at the ends of what their documentation allows:
waits that run out in tiles of one block, extreme numbers, settings per row against those of a call.

As in test_ops4_gpu.py the tolerances follow from the arithmetic and are stated at each check.
"""
import math
import time
from fractions import Fraction

import pytest
import torch

from paper_2607_01455_gb300 import Ops
from paper_2607_01455_gb300 import ember as E
from test_ops4_gpu import BF, F32, U, check_product, check_sample, gen, logits_of, rand, randn, random_table, table64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops(cuda_device):
    return Ops(cuda_device)


# ---- the product ----

@pytest.mark.parametrize("ot", [BF, F32])
@pytest.mark.parametrize("T,V,K,group", [(40, 60000, 200, 32), (300, 30000, 256, 128),
                                         # the last block alone has a stage of the scales: read by half of the warps
                                         (40, 60000, 1200, 32), (20, 60000, 2100, 64)])
def test_product_whose_waits_run_out_in_tiles_of_odd_blocks(ops, T, V, K, group, ot):
    """Several tiles a pair of CTAs, whose last block is not every widening warp's."""
    g = gen(K)
    x, t = randn(g, T, K).to(BF), random_table(g, V, K, group)
    want = ops.matmul_quant4(x, *t, group=group, dtype=ot)
    assert ops.device_status() == E.EMBER_OK
    try:
        ops.set_wait_limit_ns(1)
        for _ in range(5):
            ops.matmul_quant4(x, *t, group=group, dtype=ot)
            assert ops.device_status() == E.EMBER_ERR_TIMEOUT
    finally:
        ops.set_wait_limit_ns(0)
    assert torch.equal(ops.matmul_quant4(x, *t, group=group, dtype=ot), want) and ops.device_status() == E.EMBER_OK


@pytest.mark.parametrize("xt,ot", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("T,V,K", [(40, 60000, 200), (300, 30000, 1000), (40, 20000, 8192), (130, 600, 8192)])
def test_product_that_gave_up_has_awaited_its_copies(ops, T, V, K, xt, ot):
    """The copies in flight are all accounted for at the end: no wait for them runs into its
    own limit of two seconds, however the two CTAs of a pair were apart."""
    g = gen(K)
    x, t = randn(g, T, K).to(xt), random_table(g, V, K, 32)
    want = ops.matmul_quant4(x, *t, dtype=ot)
    assert ops.device_status() == E.EMBER_OK
    try:
        for limit in (1, 2000, 5000, 10000):  # at the first wait, and a few blocks on
            ops.set_wait_limit_ns(limit)
            for _ in range(5):
                torch.cuda.synchronize()
                t0 = time.perf_counter()
                ops.matmul_quant4(x, *t, dtype=ot)
                assert ops.device_status() in (E.EMBER_ERR_TIMEOUT, E.EMBER_OK)
                assert time.perf_counter() - t0 < 1.0
    finally:
        ops.set_wait_limit_ns(0)
    assert torch.equal(ops.matmul_quant4(x, *t, dtype=ot), want) and ops.device_status() == E.EMBER_OK


@pytest.mark.parametrize("xt", [BF, F32])
@pytest.mark.parametrize("T,V,K,group", [(1, 65536, 8192, 32), (1, 65536, 4096, 128), (3, 33, 300, 64), (1, 1, 1, 32)])
def test_product_of_few_tokens_gives_up_at_the_shortest_limit(ops, T, V, K, group, xt):
    """Every time: also where the copies come in before they are waited for."""
    g = gen(T)
    x, t = randn(g, T, K).to(xt), random_table(g, V, K, group)
    want = ops.matmul_quant4(x, *t, group=group)
    try:
        for _ in range(100):
            ops.set_wait_limit_ns(1)
            ops.matmul_quant4(x, *t, group=group)
            assert ops.device_status() == E.EMBER_ERR_TIMEOUT
            ops.set_wait_limit_ns(0)
            assert torch.equal(ops.matmul_quant4(x, *t, group=group), want) and ops.device_status() == E.EMBER_OK
    finally:
        ops.set_wait_limit_ns(0)


@pytest.mark.parametrize("xt,ot", [(BF, F32), (F32, F32), (BF, BF)])
@pytest.mark.parametrize("kw", [dict(), dict(pad_c=1)], ids=str)
@pytest.mark.parametrize("T,V,K", [(1, 333, 500), (8, 333, 500), (40, 333, 500), (130, 700, 500), (40, 256, 8192)])
def test_product_of_large_states_is_finite_where_its_results_are(ops, T, V, K, kw, xt, ot):
    """States of 1e35 and more: their products with q s, up to 3136 each, are past the floats before
    the row's scale of 1e-5 brings them back."""
    g = gen(K + T)
    got = check_product(ops, (randn(g, T, K) * 1e36).to(xt), random_table(g, V, K, 32, **kw), 32, ot)
    assert torch.isfinite(got).all()


def check_each_row(ops, x, t):
    """Against 64 bits, each output by its own row's size: fp32 states of K = 64 with twice 4 steps of
    16 products, each cut off by two ulps of the sum of magnitudes at most or a plain chain of 64 sums,
    states off by 2 u, a group's sum, two joins and the row's scale by u each: (128 + 8) u."""
    got = ops.matmul_quant4(x, *t, dtype=F32)
    q, r = table64(*t, x.shape[1], 32)
    want, terms = x.double() @ (q * r).T, x.double().abs() @ (q * r).abs().T
    assert ((got.double() - want).abs() <= 136 * U * terms).all(), ((got.double() - want).abs() / terms).max()


@pytest.mark.parametrize("kw", [dict(), dict(pad_c=1)], ids=str)
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** -30, 1.0, 2.0 ** 20])
def test_product_with_rows_of_extreme_scales(ops, T, size, kw):
    """Row scales from 2^-100 to 2^80, whose results are all within the normal floats."""
    g = gen(77)
    V, K = 180, 64
    codes, gs, _ = random_table(g, V, K, 32, **kw)
    s = torch.ldexp(1 + rand(g, V), torch.arange(-100, V - 100, device="cuda"))
    check_each_row(ops, randn(g, T, K) * size, (codes, gs, s))


@pytest.mark.parametrize("xt", [BF, F32])
@pytest.mark.parametrize("T,V,K", [(1, 200, 96), (4, 200, 2100), (40, 200, 96), (40, 200, 4096), (130, 300, 300)])
def test_states_beside_a_huge_channel(ops, T, V, K, xt):
    """A channel that no row of the table uses sets the token's power of two: other states are off by
    2^-23 of themselves (bf16: by nothing) or by 2^-39 of it."""
    g = gen(K)
    huge, at = K // 3, K // 2 + 1
    codes, gs, s = random_table(g, V, K, 32)
    byte = codes[:, huge // 2]
    codes[:, huge // 2] = (byte & 0xF0) | 8 if huge % 2 == 0 else (byte & 0x0F) | 0x80
    x = torch.zeros(T, K, device="cuda")
    x[:, huge] = (1 + rand(g, T)) * 1000
    x[:, at] = x[:, huge] * (0.5 + rand(g, T)) * torch.exp2(torch.linspace(-1, -38, T, device="cuda"))
    x = x.to(xt)
    got = ops.matmul_quant4(x, codes, gs, s, dtype=F32)
    q, r = table64(codes, gs, s, K, 32)
    x, w = x.double(), (q * r)[:, at]
    off = torch.maximum((0.0 if xt == BF else 2.0 ** -23) * x[:, at].abs(), 2.0 ** -39 * x[:, huge])
    if xt == BF:
        off[x[:, at] > 2.0 ** -31 * x[:, huge]] = 0
    # and one step that sums the two parts, cut off by two ulps at most, and the row's scale
    bound = off[:, None] * w.abs() + 5 * U * x[:, at, None] * w.abs()
    assert ((got.double() - x[:, at, None] * w).abs() <= bound).all()


@pytest.mark.parametrize("T,V", [(1, 300), (4, 300), (9, 300), (40, 300), (40, 20000), (130, 3000)])
@pytest.mark.parametrize("K", [2049, 4096])
def test_fp32_states_are_not_rounded_in_any_block(ops, T, V, K):
    """One product per sum, in the first block of K, in others and in the last: the state is off by 2 u,
    the step that sums its parts by two ulps, the row's scale by u: 7 u.  (fp16 states are off by 2^12 u.)"""
    g = gen(T)
    t = random_table(g, V, K, 32)
    q, r = table64(*t, K, 32)
    for at in (0, 255, 256, 1000, K // 2 + 3, K - 1):
        x = torch.zeros(T, K, device="cuda")
        x[:, at] = randn(g, T) * torch.exp(20 * randn(g, T))
        got = ops.matmul_quant4(x, *t, dtype=F32)
        want = x[:, at].double()[:, None] * (q * r)[:, at]
        assert ((got.double() - want).abs() <= 7 * U * want.abs()).all()


@pytest.mark.parametrize("T,V", [(4, 3000), (40, 1000), (40, 20000), (300, 2000)])
@pytest.mark.parametrize("K", [1000, 2049, 4096, 8192])
def test_fp32_sums_do_not_lose_more_with_their_length(ops, T, V, K):
    """In root mean square, as a share of |x| |w|.  A step of 16 products cuts the sum so far off by half of
    its last place on average, 0.7 2^-24 of it, and a block's sum grows with the root of its steps: 16 steps
    of a block of 256 (the small parts' are nothing beside them) lose 16 0.7 2^-24 2/3 of the block's |x| |w|
    and its sign, blocks one another's at random: 2^-21.1.  The blocks' own 32 roundings leave 2^-24 or so.  Four
    times that is the limit; fp16 states leave 2^-13, one sum over all of K = 2049 2^-18.1, of 8192 2^-16."""
    g = gen(K + T)
    x, t = randn(g, T, K), random_table(g, V, K, 64)
    q, r = table64(*t, K, 64)
    w = q * r
    err = ops.matmul_quant4(x, *t, group=64, dtype=F32).double() - x.double() @ w.T
    size = x.double().norm(dim=1)[:, None] * w.norm(dim=1)
    assert (err / size).square().mean().sqrt() <= 2.0 ** -19.1


# ---- sampling ----

@pytest.mark.parametrize("kw", [dict(), dict(top_k=5), dict(top_p=0.5), dict(min_p=0.5), dict(top_k=600, top_p=0.9)],
                         ids=str)
@pytest.mark.parametrize("T,V", [(3, 7), (20, 1001), (400, 777), (310, 8203), (2, 70001)])
@pytest.mark.parametrize("temperature", [3e29, 4e29, 2.0 ** 100])
def test_sample_of_the_lowest_logits(ops, T, V, temperature, kw):
    """Rows of -FLT_MAX and -inf, hot: what is 40 octaves below the largest is no float any
    more, and -inf stays masked; nor is anything drawn from beside a row (it starts and ends
    inside a 16-byte unit)."""
    g = gen(V)
    low = torch.finfo(F32).min
    b = torch.full((T, V + 8), math.inf, device="cuda")
    z = b[:, 3:V + 3]
    z.copy_(torch.where(rand(g, T, V) < 0.3, low, -math.inf))
    z[:, V // 2] = low
    z[::2, V // 3] = 0.9999 * low  # weights of about 1 all the same, but not quite equal
    u = rand(g, T)
    u[0] = 1 - 2.0 ** -24
    for a in (temperature, torch.full((T,), temperature, device="cuda")):
        ids, lp = check_sample(ops, z, u, temperature=a, **kw)
        assert (z.gather(1, ids[:, None]) > -math.inf).all() and torch.isfinite(lp).all()


@pytest.mark.parametrize("n", [200, 1000])
@pytest.mark.parametrize("T,V", [(310, 8000), (310, 20000), (2, 60000)])
def test_sample_top_p_cuts_behind_the_smallest_weights(ops, T, V, n):
    """n weights of 105 units and behind them n of 95, and a top-p that takes a few of the latter:
    the sum of the leading bits of the former, which go past the unit, has reached it before."""
    def logit(octave, low, high):
        """A logit about so far below a largest one of 0, and its weight in units of 2^-46: a whole
        number, what is cut off between `low` and `high`, that is odd and so stays as it is."""
        z = torch.tensor(-octave * math.log(2.0))
        while True:
            w = math.exp(z.item()) * 2.0 ** 46
            if int(w) % 2 and low < w - int(w) < high:
                return z.item(), int(w)
            z = torch.nextafter(z, torch.tensor(-100.0))

    (za, wa), (zb, wb) = logit(39.25, 0.85, 0.95), logit(39.40, 0.3, 0.7)
    # at the first's end the sum of the exact integers, and of all
    upto, mass = 2 ** 46 + n * wa, 2 ** 46 + n * (wa + wb)
    top_p = (upto + 0.4 * n) / mass  # exact to a unit
    goal = -(-Fraction(top_p) * mass // 1)
    assert upto < goal < upto + 0.8 * n and wb < wa
    kept = -(-(goal - upto) // wb)
    total = upto + kept * wb
    z = torch.full((T, V), -math.inf, device="cuda")
    b0, a0, at = 5, V // 3, V - 2
    z[:, b0:b0 + n], z[:, a0:a0 + n], z[:, at] = zb, za, 0.0
    for place, want in ((kept * wb - wb / 2, b0 + kept - 1), (kept * wb + wa / 2, a0),
                        (kept * wb + n * wa - wa / 2, a0 + n - 1), (kept * wb + n * wa + wa / 2, at)):
        ids, _ = ops.sample(z, torch.full((T,), float(place / total), device="cuda"), top_p=top_p)
        assert (ids == want).all(), (ids[:10], want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", [(40, 1000), (200, 5000), (40, 20000), (310, 20000), (3, 60000), (3, 524288)])
@pytest.mark.parametrize("shift,temperature", [(0.0, 1.0), (40.0, 0.7), (-3000.0, 0.05), (0.0, 2.0 ** 90)])
@pytest.mark.parametrize("others,kw", [(40, dict()), (40, dict(top_k=41)), (300, dict(top_k=301)),
                                       (300, dict(top_p=1 - 2.0 ** -45))], ids=str)
def test_sample_log_probabilities_of_the_rarest(ops, T, V, shift, temperature, others, kw, dtype):
    """u = 0 draws the first token, however small its weight: 18 to 38 octaves below the largest."""
    g = gen(V)
    z = torch.full((T, V), -math.inf, device="cuda")
    z[:, 5:5 + others] = (shift - temperature * randn(g, T, others).abs()).to(dtype).float()
    z[:, 7] = shift
    octaves = torch.linspace(18, 35 if "top_p" in kw else 38, T, device="cuda")  # (a top-p that keeps it)
    z[:, 0] = shift - temperature * math.log(2.0) * octaves
    z = z.to(dtype)
    ids, lp = ops.sample(z, torch.zeros(T, device="cuda"), temperature=temperature, **kw)
    d = (z.double() - z.double().amax(1, keepdim=True)) / temperature
    want = d[:, 0] - torch.logsumexp(torch.where(d > -40 * math.log(2.0), d, -math.inf), 1)
    assert (ids == 0).all()
    # |want| is 12 to 36: two ulps of the logarithm, 2^-23 36; of its argument, the exponent's rounding
    # (of at most 28: 2^-20 ln 2), two ulps of the power and one of the quotient: below 6e-6
    assert ((lp.double() - want).abs() <= 6e-6).all(), (lp.double() - want).abs().max()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", [(64, 1000), (24, 50257), (160, 4000), (310, 20000)])
def test_sample_settings_per_row_are_those_of_a_call(ops, T, V, dtype):
    """A row of a batch with settings of its own against that row alone with the same numbers, whose
    constants the host makes: the same token and the same bits of its log-probability."""
    g = gen(V)
    z, u = logits_of(g, T, V, dtype), rand(g, T)
    z[:, V - V // 50:] = -math.inf
    a = torch.exp(randn(g, T))
    a[::9] = 0
    k = torch.where(rand(g, T) < 0.5, 0, (1 + 300 * rand(g, T)).int()).int()
    p = torch.where(rand(g, T) < 0.3, 1.0, 0.5 + 0.5 * rand(g, T))
    m = torch.where(rand(g, T) < 0.5, 0.0, 0.2 * rand(g, T))
    m[1::16], p[2::16] = 1.0, 1e-3
    ids, lp = ops.sample(z, u, temperature=a, top_k=k, top_p=p, min_p=m)
    for t in range(T):
        i1, l1 = ops.sample(z[t:t + 1], u[t:t + 1], temperature=a[t].item(), top_k=k[t].item(), top_p=p[t].item(),
                            min_p=m[t].item())
        assert i1[0] == ids[t] and l1[0] == lp[t], t
