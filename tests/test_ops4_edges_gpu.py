"""The 4-bit table's operators and sampling at the ends of what their documentation allows:
waits that run out in tiles of one block, extreme numbers, settings per row against those of a call.

As in test_ops4_gpu.py the tolerances follow from the arithmetic and are stated at each check.
"""
import time

import pytest
import torch

from paper_2607_01455_gb300 import Ops
from paper_2607_01455_gb300 import ember as E
from test_ops4_gpu import BF, F32, gen, randn, random_table

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
