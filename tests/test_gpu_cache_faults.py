"""Pages that are none: whose results they reach."""
import math

import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("every", [8, 9, 10])
@pytest.mark.parametrize("D,n,Hq", [(64, 1, 8), (64, 4, 8), (128, 1, 8), (128, 9, 8)])
def test_many_short_units_beside_faulty_ones(D, n, Hq, every):
    """Units of one tile follow each other so closely that several are under way in a CTA at once: a fault reaches its own sequence alone."""
    B = 2400
    c = cp.make(B, n, Hq, 1, D, 16, [n + (i * 37) % 100 for i in range(B)], seed=D + every)
    clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
    assert not torch.isnan(clean).any()
    bad = torch.arange(B, device="cuda") % every == every - 1
    c.table[bad, 0] = c.k.shape[0] + 5
    want = clean.clone()
    want[bad] = math.nan
    for _ in range(10):
        got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~bad], clean[~bad])
    assert bv.bv_stream_status() == 0
