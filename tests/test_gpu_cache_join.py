"""The wait of the CTAs that share a unit for one another, in every kernel of the cache's attention: one of them comes when the others have given up.  The
call ends, the stream's status says so, and the counters are as before: the next calls are right, bit for bit."""
import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype,shape", [
    (BF16, (1, 1, 8, 1, 64, 16, [4000])),                        # the tensor cores: two teams, and one
    (BF16, (3, 9, 64, 8, 128, 32, [700, 9, 2000])),
    (BF16, (40, 2, 8, 4, 128, 16, [1 + 130 * i for i in range(40)])),
    (F32, (1, 1, 4, 1, 64, 16, [4000])),                         # the kernel that reads
    (F32, (40, 1, 8, 2, 128, 16, [1 + 130 * i for i in range(40)])),
    (F32, (2, 2, 4, 1, 64, 16, [3000, 40])),                     # the kernel that multiplies: 8, 16 and more rows
    (F32, (2, 4, 4, 1, 128, 16, [3000, 40])),
    (F32, (5, 9, 8, 1, 64, 16, [3000, 40, 9, 1000, 500])),
    (BF16, (5, 9, 8, 1, 36, 16, [3000, 40, 9, 1000, 500])),
])
def test_a_join_that_runs_out_ends_the_call(bv_options, dtype, shape):
    c = cp.make(*shape, dtype=dtype, seed=1)
    want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
    assert bv.bv_stream_status() == 0
    for _ in range(3):
        bv_options("wait_limit", 20000)
        bv_options("never_signal", 3)
        bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
        assert bv.bv_stream_status() == -4
        assert bv.bv_stream_status() == 0            # (reported once)
        bv.bv_set_option("never_signal", 0)
        # (the waits are as short still: those of a call that nobody is late for do not run out)
        assert torch.equal(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens), want) and bv.bv_stream_status() == 0
        bv.bv_set_option("wait_limit", 0)
        for _ in range(2):
            assert torch.equal(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens), want)
    # (neither do they where a unit is one CTA's: nobody is late)
    bv_options("never_signal", 3)
    one = cp.make(1, 1, 4, 4, 64, 16, [20], dtype=dtype, seed=2)
    bv.bv_cache_attend(one.q, one.k, one.v, one.table, one.lens)
    assert bv.bv_stream_status() == 0
