"""Waits of the cache's attention that run out: the scores are never announced, so every wait behind them gives up after a few thousand
polls; the call ends, the stream's status says so, and the next call is right."""
import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 1, 8, 8, 64, 16, [1000]), (3, 9, 64, 8, 128, 32, [700, 9, 2000]), (40, 2, 8, 4, 128, 16, [1 + 53 * i for i in range(40)])])
def test_a_wait_that_runs_out_ends_the_call(bv_options, shape):
    c = cp.make(*shape, seed=1)
    want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
    assert bv.bv_stream_status() == 0
    bv_options("wait_limit", 3000)
    bv_options("never_signal", 1)
    bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    assert bv.bv_stream_status() == -4
    assert bv.bv_stream_status() == 0            # (reported once)
    bv.bv_set_option("never_signal", 0)
    bv.bv_set_option("wait_limit", 0)
    for _ in range(3):
        assert torch.equal(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens), want)
    assert bv.bv_stream_status() == 0
