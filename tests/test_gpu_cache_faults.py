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


# (n, Hq, Hkv, D, page, lengths): blocks of one and of several tiles of query rows in every kernel, whole units and units that several CTAs have
SHAPES = [
    (1, 4, 1, 64, 16, [300, 40]),
    (2, 2, 1, 64, 16, [300, 34]),
    (9, 16, 2, 64, 16, [150, 2000]),
    (40, 8, 1, 128, 16, [600, 47]),                              # 320 rows a head
    (90, 4, 2, 64, 24, [100, 90, 500] + [95] * 40),
    (12, 16, 1, 128, 200, [210, 5000]),                          # pages longer than a tile
    (20, 6, 1, 80, 48, [30, 1500]),
    (3, 4, 1, 33, 5, [19, 200]),                                 # off the tensor cores
    (11, 4, 1, 192, 7, [40, 300]),
    (2, 1, 1, 256, 16, [17, 600]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (25, 3), (130, 20)])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_page_that_is_none_is_nan_for_the_rows_that_see_it(shape, window, sinks, dtype):
    n, Hq, Hkv, D, page, lens = shape
    B = len(lens)
    c = cp.make(B, n, Hq, Hkv, D, page, lens, dtype=dtype, seed=n)
    good = c.table.clone()
    clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window, sinks=sinks).clone()
    held = [cp.ceil_div(L, page) for L in lens]
    faults = [[h - 1 for h in held],                             # the last page: the block's later tokens
              [0] * B,                                           # the first: everybody, or with a window those whose sinks it has
              [max(0, L - n - 10) // page for L in lens],        # one that the first tokens' windows have and the last ones' do not
              [max(0, L - n // 2 - 1) // page for L in lens]]
    for at in faults:
        for no_page in (-1, c.k.shape[0], 2**31 - 1):
            c.table.copy_(good)
            for b in range(0, B, 2):
                c.table[b, at[b]] = no_page
            got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window, sinks=sinks)
            lost = torch.zeros((B, n), dtype=torch.bool)
            for b in range(0, B, 2):
                for t in range(n):
                    lost[b, t] = any(j // page == at[b] for j in cp.visible(lens[b] - n + t, window, sinks, lens[b]))
            assert torch.isnan(got[lost]).all() and torch.equal(got[~lost], clean[~lost]), (at, no_page)
    assert bv.bv_stream_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_lay_where_a_page_is_none_does_not_count(dtype):
    """The places of such a page hold what an earlier tile, or an earlier call, left there: infinities and NaN, here."""
    for n, Hq, D in ((12, 8, 64), (12, 8, 128), (30, 8, 128), (6, 2, 36)):
        foul = cp.make(8, n, Hq, 1, D, 16, [900] * 8, dtype=dtype, seed=1)
        foul.k.fill_(math.nan)
        foul.v.fill_(math.inf)
        c = cp.make(40, n, Hq, 1, D, 16, [n + 16 * (i % 4) + 5 for i in range(40)], dtype=dtype, seed=2)
        clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
        for b, L in enumerate(c.lens.tolist()):
            c.table[b, (L - 1) // 16] = -1
        lost = torch.zeros((40, n), dtype=torch.bool)
        for b, L in enumerate(c.lens.tolist()):
            for t in range(n):
                lost[b, t] = (L - n + t) // 16 == (L - 1) // 16
        for _ in range(3):
            bv.bv_cache_attend(foul.q, foul.k, foul.v, foul.table, foul.lens)
            got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
            assert torch.isnan(got[lost]).all() and torch.equal(got[~lost], clean[~lost])
