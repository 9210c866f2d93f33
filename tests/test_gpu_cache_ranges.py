"""The paged cache at the ends of the ranges that its calls accept."""
import random

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


def test_sequences_that_ask_for_all_pages_of_the_largest_cache():
    """1024 sequences of one-token pages, each of which would take the whole pool: the first gets it, the second half's sums are no fewer for
    that.  With nothing free only those that ask for nothing are served."""
    B, P = 1024, 2**22 - 2
    if torch.cuda.mem_get_info()[0] < 4 * B * P + (1 << 32):
        pytest.skip("a table of 17 GB")
    table = torch.empty((B, P), dtype=torch.int32, device="cuda")
    table[:, :2] = table[:, -2:] = -1
    lens, refs = torch.zeros((B,), dtype=torch.int32, device="cuda"), torch.zeros((P,), dtype=torch.int32, device="cuda")
    new, copies = bv.bv_pages_extend(table, lens, refs, 1, P)
    assert new.tolist() == [P] + [-1] * (B - 1) and (copies == -1).all()
    assert lens.tolist() == [P] + [0] * (B - 1) and (refs == 1).all()
    assert torch.equal(table[0], torch.arange(P, dtype=torch.int32, device="cuda")) and (table[1:, :2] == -1).all() and (table[1:, -2:] == -1).all()
    lens.zero_()
    asked = torch.full((B,), P, dtype=torch.int32, device="cuda")
    asked[::7] = 0
    new, _ = bv.bv_pages_extend(table, lens, refs, 1, P, asked)
    assert new.tolist() == [0 if b % 7 == 0 else -1 for b in range(B)] and (lens == 0).all() and (refs == 1).all()
    # half of the pool free, the second half of the batch asks for it
    refs[1::2] = 0
    asked.fill_(0)
    asked[600:] = P // 2
    new, _ = bv.bv_pages_extend(table, lens, refs, 1, P, asked)
    assert new.tolist() == [0] * 600 + [P // 2] + [-1] * 423 and (refs == 1).all()
    assert torch.equal(table[600, :P // 2], torch.arange(1, P, 2, dtype=torch.int32, device="cuda"))


def cut_back(lens, table, refs, page, keep, n, n_new):
    """What bv_pages_truncate leaves, by its contract: of the m newest tokens, n_new[b] held to 0 .. n, the first keep[b] stay."""
    lens, table, refs = list(lens), [list(r) for r in table], list(refs)
    for b, L in enumerate(lens):
        m = min(L, max(0, min(n, n_new[b])))
        lens[b] = L - m + max(0, min(m, keep[b]))
        for j in range(cp.ceil_div(lens[b], page), cp.ceil_div(L, page)):
            refs[table[b][j]] -= 1
            table[b][j] = -1
    return lens, table, refs


def test_a_block_that_is_cut_back_has_n_tokens_at_most():
    """More in n_new than n is n, as for the attention and for storing: tokens before the block stay."""
    table, lens, refs = i32([[0, 1, 2], [3, 4, -1], [5, -1, -1]]), i32([10, 8, 2]), i32([1] * 6)
    bv.bv_pages_truncate(table, lens, refs, 4, i32([1, 0, 0]), 3, i32([9, 2**31 - 1, 4]))
    assert lens.tolist() == [8, 5, 0]
    assert table.tolist() == [[0, 1, -1], [3, 4, -1], [-1, -1, -1]] and refs.tolist() == [1, 1, 0, 1, 1, 0]


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("page", [1, 3, 16])
def test_blocks_cut_back_whatever_n_new_says(seed, page):
    rng = random.Random(seed)
    B, n = 40, rng.choice((1, 2, 5, 9))
    lens = [rng.choice((0, 1, n, rng.randint(0, 6 * page))) for _ in range(B)]
    c = cp.make(B, 1, 1, 1, 4, page, lens, dtype=F32, seed=seed)
    keep, new = [rng.randint(-1, n + 3) for _ in range(B)], [rng.randint(-2, n + 3) for _ in range(B)]
    want = cut_back(lens, c.table.tolist(), c.refs.tolist(), page, keep, n, new)
    bv.bv_pages_truncate(c.table, c.lens, c.refs, page, i32(keep), n, i32(new))
    assert (c.lens.tolist(), c.table.tolist(), c.refs.tolist()) == want


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,Hq,D", [(1, 4, 64), (1, 8, 128), (9, 8, 128), (3, 4, 36)])
@pytest.mark.parametrize("score", [1e5, 1e6, 3e7, 1e9, 3e10, 1e14, 1e25, 1e33])
def test_scores_of_every_size(score, n, Hq, D, dtype):
    """Two keys of the same large score, tiles and CTAs apart, among others far below: the mean of their values (weights of one and of nothing, so no
    rounding but the result's).  Then keys that differ by little in all of them: some weighted mean of what a row sees."""
    L = 3000
    c = cp.make(2, n, Hq, 1, D, 16, [L, 700], dtype=dtype, seed=24)
    size = (score / D ** 0.5) ** 0.5                             # of q's and of the keys' elements: the scaled score is their product times sqrt(D)
    c.q.fill_(size)
    c.k.fill_(-size)
    for sign in (1, -1):
        c.v[:, :, :, :] = 7.0
        for b, tops in enumerate(((130, 2700), (0, 127))):
            for j, val in zip(tops, (1.0, 3.0)):
                at = (c.table[b, j // 16].item(), slice(None), j % 16)
                c.k[at], c.v[at] = size * sign, val
        got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, scale=sign * D ** -0.5)
        assert (got == 2.0).all(), sign
        c.k.mul_(-1)
    g = torch.Generator().manual_seed(25)
    c.k.copy_((size * (1 + 0.05 * torch.randn(c.k.shape, generator=g))).to(dtype))
    c.v.copy_(torch.rand(c.v.shape, generator=g).to(dtype))
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    assert (got >= 0).all() and (got <= 1).all()
    assert bv.bv_stream_status() == 0


@pytest.mark.parametrize("dtype,D", [(F32, 2**29), (BF16, 2**30 - 8)])
def test_rows_of_2_to_the_31_bytes(dtype, D):
    """Stored in a page and copied to another (one pool for keys and values: the same ones)."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("four rows of 2 GB")
    pool = torch.zeros((3, 1, 1, D), dtype=dtype, device="cuda")
    row = torch.zeros((1, 1, 1, D), dtype=dtype, device="cuda")
    row.view(-1)[::1001] = 3.0
    row.view(-1)[-1], row.view(-1)[0] = 5.0, 7.0
    table, lens = i32([[1]]), i32([1])
    bv.bv_cache_append(row, row, pool, pool, table, lens)
    assert torch.equal(pool[1], row[0]) and not pool[0].any() and not pool[2].any()
    bv.bv_pages_copy(pool, pool, i32([[1, 0]]))
    assert torch.equal(pool[0], row[0]) and torch.equal(pool[1], row[0]) and not pool[2].any()
