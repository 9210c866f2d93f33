"""Attention over the paged cache against the definition in 64 bits, with bounds by arithmetic (cache_plain.attend)."""
import math

import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def check(c, n_new=None, window=0, sinks=0, scale=None, out=None):
    before = None if out is None else out.clone()
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, n_new=n_new, window=window, sinks=sinks, scale=scale, out=out)
    assert bv.bv_stream_status() == 0 and bv.bv_last_launch_count() == 1
    want, bound, written = cp.attend(c.q, c.k, c.v, c.table, c.lens, n_new, scale, window, sinks, 8 if c.q.dtype == BF16 else 24)
    g = got.double().cpu()
    rows = written[:, :, None, None].expand_as(g)
    assert torch.equal(torch.isnan(g) & rows, torch.isnan(want) & rows)
    fine = rows & ~torch.isnan(want)
    off = (g - want).abs()
    worst = (off - bound)[fine].max().item() if fine.any() else 0.0
    assert worst <= 0, "off by %.3g more than the bound" % worst
    rest = (torch.zeros_like(g) if before is None else before.double().cpu())[~rows]
    assert torch.equal(g[~rows], rest)
    return got


# (B, n, Hq, Hkv, D, page, lengths)
SHAPES = [
    (1, 1, 1, 1, 64, 16, [1]),                                   # one token, one key
    (1, 1, 8, 8, 64, 16, [1000]),
    (3, 1, 8, 2, 128, 16, [1, 127, 129]),                        # around a tile
    (4, 1, 4, 4, 128, 32, [128, 256, 255, 257]),
    (2, 9, 64, 8, 128, 32, [9, 700]),                            # 72 rows a head; a block that is its whole sequence
    (5, 5, 10, 2, 64, 64, [5, 6, 64, 65, 333]),
    (3, 3, 7, 1, 80, 24, [3, 24, 500]),                          # odd sizes
    (2, 17, 16, 1, 128, 128, [17, 900]),                         # 272 rows a head
    (2, 2, 6, 3, 96, 192, [191, 400]),                           # pages longer than a tile
    (2, 4, 4, 2, 72, 256, [256, 1000]),
    (2, 3, 4, 1, 33, 5, [4, 77]),                                # nothing is a whole vector
    (2, 2, 4, 2, 200, 8, [30, 90]),
    (2, 2, 2, 1, 256, 16, [100, 41]),
    (1, 1, 32, 32, 128, 8, [300]),
    (2, 33, 4, 4, 128, 16, [33, 210]),
    (2, 1, 128, 1, 64, 1, [1, 50]),                              # a page a token
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_attention_is_the_definition(shape, dtype, layout):
    check(cp.make(*shape, dtype=dtype, layout=layout, seed=len(shape[6])))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (64, 4), (127, 17), (128, 0), (300, 200), (2**31 - 1, 3)])
def test_windows_and_sinks(dtype, window, sinks):
    check(cp.make(4, 6, 8, 2, 64, 16, [6, 90, 513, 1300], dtype=dtype, seed=3), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_work_of_one_sequence_is_joined(dtype):
    check(cp.make(1, 1, 8, 1, 128, 64, [20011], dtype=dtype, seed=5, q_scale=4.0))
    check(cp.make(2, 9, 8, 1, 64, 16, [5000, 12], dtype=dtype, seed=6, q_scale=4.0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,Hq,Hkv", [(1, 2, 1), (1, 8, 4), (1, 16, 2), (5, 6, 1), (9, 16, 2), (13, 16, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 7)])
def test_fewer_units_than_ctas(dtype, n, Hq, Hkv, window, sinks):
    """Sequences of all lengths whose heads are shared out to the CTAs whole, in parts of their own, or as the list is cut."""
    for lens in ([n], [700, n, 64], [1 + 130 * (i * 11 % 29) for i in range(29)], [30, 4000] + [20] * 30):
        check(cp.make(len(lens), n, Hq, Hkv, 64, 16, lens, dtype=dtype, seed=len(lens)), window=window, sinks=sinks)
    lens = [700, n, 64, 128]
    c = cp.make(4, n, Hq, Hkv, 64, 16, lens, dtype=dtype, seed=22)
    check(c, n_new=torch.tensor([n, 0, 1, n // 2], dtype=torch.int32, device="cuda"), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_blocks_of_different_lengths_leave_the_other_rows(dtype):
    c = cp.make(6, 5, 8, 2, 64, 16, [40, 3, 0, 100, 17, 200], dtype=dtype, seed=7)
    new = torch.tensor([5, 3, 0, 1, -2, 9], dtype=torch.int32, device="cuda")
    out = torch.full_like(c.q, 7.0)
    check(c, n_new=new, out=out)
    check(c, n_new=new, out=torch.full_like(c.q, 7.0), window=8, sinks=2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing_are_zero(dtype):
    # blocks longer than their sequences: the first tokens lie before position 0
    c = cp.make(3, 4, 4, 2, 64, 16, [0, 1, 3], dtype=dtype, seed=8)
    got = check(c)
    assert (got[0] == 0).all() and (got[1, :3] == 0).all() and (got[1, 3] != 0).any() and (got[2, 0] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_what_is_not_seen_does_not_count(dtype, value, window, sinks):
    """Rows behind the sequence, pages of nobody, positions out of the window, and the block's later tokens for its earlier ones."""
    page, lens, n = 16, [37, 150, 129], 4
    c = cp.make(3, n, 4, 2, 64, page, lens, dtype=dtype, seed=9)
    clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window, sinks=sinks).clone()
    named = set(x for row in c.table.cpu().tolist() for x in row if x >= 0)
    for p in range(c.k.shape[0]):
        if p not in named:
            c.k[p], c.v[p] = value, value
    for b, L in enumerate(lens):
        for j in range(L, cp.ceil_div(L, page) * page):
            c.k[c.table[b, j // page].item(), :, j % page], c.v[c.table[b, j // page].item(), :, j % page] = value, value
        for j in range(L):
            if window and j >= sinks and j <= L - n - window:
                p = c.table[b, j // page].item()
                c.k[p, :, j % page], c.v[p, :, j % page] = value, value
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window, sinks=sinks)
    assert torch.equal(got, clean)
    # the newest token's key and value: only the newest token's result may change
    for b, L in enumerate(lens):
        p = c.table[b, (L - 1) // page].item()
        c.v[p, :, (L - 1) % page, ::3] = value
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window, sinks=sinks)
    assert torch.equal(got[:, :n - 1], clean[:, :n - 1])
    last, was = got[:, n - 1], clean[:, n - 1]
    if math.isnan(value):
        assert torch.isnan(last[..., ::3]).all()
    else:
        assert (last[..., ::3] == value).all()
    rest = torch.ones(64, dtype=torch.bool)
    rest[::3] = False
    assert torch.equal(last[..., rest], was[..., rest])
    for b, L in enumerate(lens):
        p = c.table[b, (L - 1) // page].item()
        c.k[p, :, (L - 1) % page] = math.nan
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window, sinks=sinks)
    assert torch.equal(got[:, :n - 1], clean[:, :n - 1]) and torch.isnan(got[:, n - 1]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_value_that_leaves_an_old_token_s_window_is_seen_by_the_earlier_tokens_only(dtype):
    page, L, n, window = 16, 200, 5, 30
    c = cp.make(1, n, 2, 1, 64, page, [L], dtype=dtype, seed=10)
    clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window).clone()
    j = L - n - window + 1 + 2                # seen by tokens 0, 1, 2 of the block
    c.v[c.table[0, j // page].item(), :, j % page] = math.inf
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=window)
    assert (got[0, :3] == math.inf).all() and torch.equal(got[0, 3:], clean[0, 3:])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_faults_are_a_sequence_s_own(dtype):
    c = cp.make(5, 2, 4, 2, 64, 16, [100, 100, 100, 100, 100], dtype=dtype, seed=11)
    clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
    c.table[1, 3] = c.k.shape[0]
    c.table[2, 6] = -1
    c.lens[3] = 16 * c.table.shape[1] + 1
    c.lens[4] = -5
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    assert torch.equal(got[0], clean[0]) and torch.isnan(got[1:]).all()
    # a page that is none, out of everybody's sight
    c.table[1, 0] = -7
    c.table[1, 3] = 0
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=40)
    assert not torch.isnan(got[:2]).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_far_apart(dtype):
    """Scores that differ by hundreds, rising along the sequence, so that the reference has to move again and again."""
    c = cp.make(1, 3, 4, 1, 64, 16, [700], dtype=dtype, seed=12)
    c.q.fill_(1.0)
    flat = torch.arange(700, device="cuda").float() * 0.07
    for j in range(700):
        c.k[c.table[0, j // 16].item(), :, j % 16] = flat[j].to(dtype)
    check(c, scale=0.5)
    check(c, scale=-0.5)
    check(c, scale=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,Hq", [(1, 4), (9, 8)])
def test_a_first_score_far_from_the_others(dtype, n, Hq):
    """The first key, or the last of its tile, far below, far above and beside the others; values near the type's largest."""
    for factor in (-30.0, -8.0, 0.0, 8.0, 30.0):
        c = cp.make(2, n, Hq, 1, 64, 16, [1000, 140], dtype=dtype, seed=23)
        c.q[..., 0] = 2.0
        for b in range(2):
            for j in (0, 127, 128):
                c.k[c.table[b, j // 16].item(), :, j % 16, 0] = factor * 8
        c.v *= 2.0 ** 100
        check(c)
        check(c, window=60, sinks=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,Hq,D", [(1, 2, 64), (3, 4, 64), (9, 16, 128), (2, 2, 33)])
def test_a_row_of_scores_of_minus_infinity(dtype, n, Hq, D):
    """Such a score weighs nothing beside others; a row of nothing else is 0 / 0."""
    c = cp.make(3, n, Hq, 1, D, 16, [40, 900, n], dtype=dtype, seed=18)
    c.q[..., 0] = 1.0
    clean = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
    c.k[..., 0] = -math.inf
    assert torch.isnan(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)).all()
    # one key of the last sequence's that is not: the rows that see it have its value, those before it do not
    at = (c.table[2, (n - 1) // 16].item(), slice(None), (n - 1) % 16, 0)
    c.k[at] = 1.0
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    assert torch.isnan(got[:2]).all() and torch.isnan(got[2, :n - 1]).all()
    assert torch.equal(got[2, n - 1], c.v[c.table[2, (n - 1) // 16].item(), 0, (n - 1) % 16].expand(Hq, D))
    assert not torch.isnan(clean).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignment(dtype):
    c = cp.make(3, 3, 4, 2, 64, 16, [50, 300, 129], dtype=dtype, seed=13)
    ref = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    # q and out as slices of wider tensors, the pool as every second page of a larger one
    wide = torch.zeros((3, 5, 4, 80), dtype=dtype, device="cuda")
    q = wide[:, 1:4, :, 8:72]
    q.copy_(c.q)
    outs = torch.zeros((4, 3, 3, 64), dtype=dtype, device="cuda").permute(1, 2, 0, 3)
    big = torch.zeros((2 * c.k.shape[0],) + tuple(c.k.shape[1:]), dtype=dtype, device="cuda")
    big[::2] = c.k
    got = bv.bv_cache_attend(q, big[::2], c.v, c.table, c.lens, out=outs)
    assert torch.equal(got, ref)
    # a pool one element off every boundary
    off = torch.zeros((c.k.numel() + 1,), dtype=dtype, device="cuda")[1:].view(c.k.shape)
    off.copy_(c.k)
    c.k = off
    check(c)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 9])
def test_pools_whose_heads_or_pages_are_one(dtype, n):
    c = cp.make(2, n, 8, 2, 64, 16, [50, 300], dtype=dtype, seed=20)
    k, v = c.k, c.v
    c.k, c.v = k[:, :1].expand_as(k), v[:, :1].expand_as(v)
    check(c)
    c.k, c.v = k, v[3:4].expand_as(v)
    check(c)


@pytest.mark.parametrize("page", [8, 24, 40, 48, 56, 72, 80, 96, 104, 112, 120, 136, 160, 192, 200, 320, 1000])
@pytest.mark.parametrize("window,sinks", [(0, 0), (130, 50)])
def test_every_kind_of_page(page, window, sinks):
    """Pages that divide a tile, that tiles go across in smaller boxes, or that are several tiles themselves."""
    for n, D in ((1, 128), (9, 64)):
        c = cp.make(4, n, 16, 2, D, page, [n, 127, page, 900], seed=page)
        clean = check(c, window=window, sinks=sinks).clone()
        # rows behind the sequences, and pages of nobody
        for b, L in enumerate([n, 127, page, 900]):
            for j in range(L, cp.ceil_div(L, page) * page):
                c.k[c.table[b, j // page].item(), :, j % page] = c.v[c.table[b, j // page].item(), :, j % page] = math.nan
        c.k[c.refs == 0] = c.v[c.refs == 0] = math.nan
        assert torch.equal(check(c, window=window, sinks=sinks), clean)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [5, 7, 8, 12, 16, 17, 24, 40, 48, 49, 64, 65, 96, 128])
@pytest.mark.parametrize("D", [36, 64, 128, 192])
def test_every_number_of_rows(dtype, rows, D):
    check(cp.make(3, rows // 8 if rows % 8 == 0 else rows, 8 if rows % 8 == 0 else 1, 1, D, 16, [130, 700, 64], dtype=dtype, seed=21))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_same_bits_every_time(dtype):
    c = cp.make(9, 5, 16, 2, 128, 16, [2000, 5, 700, 31, 999, 1500, 64, 63, 3000], dtype=dtype, seed=14)
    ref = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    for _ in range(20):
        assert torch.equal(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens), ref)


def test_two_streams_and_a_graph():
    c = cp.make(4, 3, 8, 2, 128, 16, [500, 900, 20, 333], seed=15)
    ref = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens).clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(c.q) for _ in streams]
    for _ in range(10):
        for s, o in zip(streams, outs):
            bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, out=o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    # captured once, replayed as the sequences grow
    out = torch.zeros_like(c.q)
    s = streams[0]
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, out=out, stream=s)
    for lens in ([500, 900, 20, 333], [3, 16, 17, 300], [496, 1, 3, 128]):
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.zero_()
        g.replay()
        want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_offsets_beyond_32_bits():
    """Pages that lie beyond 2^31 elements (and 2^32 bytes) of their pool."""
    P = (1 << 31) // (16 * 128) + 4
    pool = torch.empty((P, 1, 16, 128), dtype=BF16, device="cuda")
    c = cp.make(1, 2, 4, 1, 128, 16, [40], seed=16)
    far = torch.tensor([P - 1, P - 3, 1], dtype=torch.int32, device="cuda")
    for to, at in zip(far.tolist(), c.table[0].tolist()):
        pool[to] = c.k[at]
    want = bv.bv_cache_attend(c.q, c.k, c.k, c.table, c.lens).clone()
    got = bv.bv_cache_attend(c.q, pool, pool, far[None].contiguous(), c.lens)
    assert torch.equal(got, want)
    # (keys and values into the one pool: the same ones)
    bv.bv_cache_append(c.k_new, c.k_new, pool, pool, far[None].contiguous(), c.lens)
    assert torch.equal(pool[1, 0, 6:8], c.k_new[0, :, 0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 9])
def test_positions_next_to_2_to_the_31(dtype, n):
    """The longest sequence there is, on one page named again and again, seen through a window: what a shorter one on that page sees.  A token
    more is a length that is none."""
    page, most = 1 << 20, 2**31 - 1024
    c = cp.make(1, n, 2, 1, 16, page, [page - 1024], dtype=dtype, seed=19, spare=0)
    want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, window=200, sinks=5)
    table = c.table.expand(1, 2048).contiguous()
    lens = torch.tensor([most], dtype=torch.int32, device="cuda")
    got = bv.bv_cache_attend(c.q, c.k, c.v, table, lens, window=200, sinks=5)
    assert torch.equal(got, want) and not torch.isnan(got).any()
    assert torch.isnan(bv.bv_cache_attend(c.q, c.k, c.v, table, lens + 1, window=200, sinks=2000)).all()
    k = c.k.clone()
    bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, table, lens + 1)
    assert torch.equal(c.k, k)
    bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, table, lens)
    assert torch.equal(c.k[0, 0, page - 1024 - n:page - 1024], c.k_new[0, :, 0]) and bv.bv_stream_status() == 0


def test_many_short_sequences():
    lens = [1 + (i * 37) % 50 for i in range(700)]
    check(cp.make(700, 1, 2, 1, 64, 16, lens, seed=17))
