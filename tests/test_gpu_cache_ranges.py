"""The paged cache at the ends of the ranges that its calls accept."""
import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_lowest_lengths_have_no_tokens(dtype):
    """A length of -2^31 and a little more: from which a block's length is not to be subtracted."""
    n = 5
    c = cp.make(6, n, 4, 2, 64, 16, [40] * 6, dtype=dtype, seed=1)
    for new in (None, i32([n, 1, 2, n, 3, n])):
        c.lens[:5] = i32([-2**31, -2**31 + 1, -2**31 + n - 1, -2**31 + n, -1])
        k, v = c.k.clone(), c.v.clone()
        for t in range(n):
            p = 40 - n + t
            k[c.table[5, p // 16].item(), :, p % 16] = c.k_new[5, t]
            v[c.table[5, p // 16].item(), :, p % 16] = c.v_new[5, t]
        bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, c.table, c.lens, n_new=new)
        assert torch.equal(c.k, k) and torch.equal(c.v, v)
        out = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
        assert torch.isnan(out[:5]).all() and not torch.isnan(out[5]).any()
        before = c.table.clone(), c.lens.clone(), c.refs.clone()
        bv.bv_pages_truncate(c.table, c.lens, c.refs, 16, i32([0] * 5 + [9]), 3)
        assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.lens, c.refs)))
        got, _ = bv.bv_pages_extend(c.table, c.lens, c.refs, 16, 1, i32([1, 1, 1, 1, 1, 0]))
        assert got.tolist() == [-1] * 5 + [0]
    assert bv.bv_stream_status() == 0
