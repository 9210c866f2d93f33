"""Storing in, and the bookkeeping of, the paged cache: integers and copies, exact."""
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
@pytest.mark.parametrize("D,page,layout", [(64, 16, "heads"), (128, 24, "tokens"), (33, 5, "heads"), (20, 1, "tokens")])
def test_append(dtype, D, page, layout):
    c = cp.make(5, 7, 4, 2, D, page, [7, 100, 3, 0, 40], dtype=dtype, layout=layout, seed=1)
    c.table[4, 39 // page] = -1                # (its last tokens have no page: passed over)
    new = i32([7, 4, 7, 7, 7])
    k, v = c.k.clone(), c.v.clone()
    for b, (L, m) in enumerate(zip(c.lens.tolist(), new.tolist())):
        for t in range(m):
            p = L - m + t
            if p < 0 or c.table[b, p // page] < 0:
                continue
            k[c.table[b, p // page].item(), :, p % page] = c.k_new[b, t]
            v[c.table[b, p // page].item(), :, p % page] = c.v_new[b, t]
    bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, c.table, c.lens, n_new=new)
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    # all of a wider tensor's tokens, lengths that are none
    wide = torch.randn((5, 9, 3, D), device="cuda").to(dtype)
    c.lens[1], c.lens[2] = -3, c.table.shape[1] * page + 1
    c.lens[3] = 0
    k, v = c.k.clone(), c.v.clone()
    for t in range(2):
        for b in (0, ):
            p = c.lens[b].item() - 2 + t
            k[c.table[b, p // page].item(), :, p % page] = wide[b, 3 + t, 1:]
            v[c.table[b, p // page].item(), :, p % page] = wide[b, 5 + t, :2]
    bv.bv_cache_append(wide[:, 3:5, 1:], wide[:, 5:7, :2], c.k, c.v, c.table, c.lens, n_new=i32([2, 2, 2, 2, 0]))
    assert torch.equal(c.k, k) and torch.equal(c.v, v)


def same(book, table, lens, refs):
    assert lens.tolist() == book.lens
    assert refs.tolist() == book.refs
    assert table.tolist() == book.table


def small_cache(rng, B, page, width, P):
    """Sequences of all lengths, some sharing pages, on pages in no order."""
    order = list(range(P))
    rng.shuffle(order)
    table, lens, refs = [[-1] * width for _ in range(B)], [0] * B, [0] * P
    for b in range(B):
        if b and rng.random() < 0.4:                           # a branch of an earlier one, perhaps cut back
            a = rng.randrange(b)
            lens[b] = rng.randint(0, lens[a])
            for j in range(cp.ceil_div(lens[b], page)):
                table[b][j] = table[a][j]
                refs[table[b][j]] += 1
            continue
        lens[b] = rng.choice((0, 1, page, page + 1, rng.randint(0, width * page)))
        held = cp.ceil_div(lens[b], page)
        if held > len(order):
            lens[b] = held = 0
        for j in range(held):
            table[b][j] = order.pop()
            refs[table[b][j]] += 1
    return i32(table), i32(lens), i32(refs)


@pytest.mark.parametrize("seed", range(12))
def test_a_random_walk_of_all_of_them(seed):
    """Extend, truncate, fork, compact with copies, in random order, against lists; and what the pages hold goes with them."""
    rng = random.Random(seed)
    page, width = rng.choice((1, 3, 16)), rng.choice((2, 9))
    B, P = rng.choice((1, 5, 40)), rng.choice((1, 7, 60, 300))
    table, lens, refs = small_cache(rng, B, page, width, P)
    book = cp.Book(table, lens, refs, page)
    # every page holds a number of its own; a token's value is what its page and row held when it was appended
    k = torch.arange(P * page, device="cuda").float().view(P, 1, page, 1).expand(P, 1, page, 4).contiguous()
    v = -k.clone()

    def contents():
        kk = k[:, 0, :, 0].cpu()
        return [[kk[book.table[b][j // page], j % page].item() for j in range(book.lens[b])] for b in range(B)]

    held = contents()
    for step in range(14):
        what = rng.choice(("extend", "extend", "truncate", "fork", "compact"))
        if what == "extend":
            n = rng.choice((1, 2, 5, 40))
            new = None if rng.random() < 0.3 else [rng.choice((0, 0, 1, n, rng.randint(-1, n + 1))) for _ in range(B)]
            got, copies = bv.bv_pages_extend(table, lens, refs, page, n, None if new is None else i32(new))
            want, wcopies = book.extend(n, new)
            assert got.tolist() == want and copies.tolist() == wcopies
            bv.bv_pages_copy(k, v, copies)
            # (the new tokens: numbers of their own, through the table)
            kk = torch.full((B, n, 1, 4), float(step), device="cuda")
            bv.bv_cache_append(kk, -kk, k, v, table, lens, n_new=got)
            held = [h + [float(step)] * max(0, m) for h, m in zip(held, want)]
        elif what == "truncate":
            n = rng.choice((0, 1, 5))
            keep = [rng.randint(-1, 9) if rng.random() < 0.7 else 2**31 - 1 for _ in range(B)]
            new = None if n == 0 or rng.random() < 0.5 else [rng.randint(-1, n) for _ in range(B)]
            bv.bv_pages_truncate(table, lens, refs, page, i32(keep), n, None if new is None else i32(new))
            book.truncate(keep, n, new)
            held = [h[:L] for h, L in zip(held, book.lens)]
        elif what == "fork":
            F = rng.randint(1, B)
            src, dst = [rng.randint(-1, B) for _ in range(F)], [rng.randint(-1, B) for _ in range(F)]
            ok = bv.bv_pages_fork(table, lens, refs, page, i32(src), i32(dst))
            assert ok.tolist() == book.fork(src, dst)
            was = [list(h) for h in held]
            for s, d, o in zip(src, dst, ok.tolist()):
                if o == 0:
                    held[d] = list(was[s])
        else:
            moves, count = bv.bv_pages_compact(table, lens, refs, page)
            wmoves, wcount = book.compact()
            assert count.tolist() == [wcount] and moves.tolist() == wmoves
            bv.bv_pages_copy(k, v, moves, count)
            used = sum(1 for r in book.refs if r)
            assert all(r > 0 for r in book.refs[:used])
        same(book, table, lens, refs)
        assert contents() == held
        assert torch.equal(v, -k)
    assert bv.bv_stream_status() == 0


@pytest.mark.parametrize("P", [8191, 8192, 8193, 30000, 100001])
def test_large_pools(P):
    """Several CTAs look at the counts; the ends of their regions."""
    rng = random.Random(P)
    refs = [0 if rng.random() < 0.3 else 1 for _ in range(P)]
    refs[0], refs[-1] = 0, 0
    used = [p for p in range(P) if refs[p]]
    B, page = 60, 16
    width = cp.ceil_div(P, B) + 3
    table, lens = [[-1] * width for _ in range(B)], [0] * B
    for b in range(B):
        part = used[b::B]
        table[b][:len(part)] = part
        lens[b] = max(0, len(part) * page - rng.randrange(page))
    t, ln, rf = i32(table), i32(lens), i32(refs)
    book = cp.Book(t, ln, rf, page)
    for n in (1, 700):
        got, copies = bv.bv_pages_extend(t, ln, rf, page, n)
        want, wcopies = book.extend(n)
        assert got.tolist() == want and copies.tolist() == wcopies
        same(book, t, ln, rf)
    keep = [rng.choice((0, 50, 10**6)) for _ in range(B)]
    bv.bv_pages_truncate(t, ln, rf, page, i32(keep))
    book.truncate(keep)
    same(book, t, ln, rf)
    moves, count = bv.bv_pages_compact(t, ln, rf, page)
    wmoves, wcount = book.compact()
    assert count.tolist() == [wcount] and moves.tolist() == wmoves
    same(book, t, ln, rf)


def test_running_out_of_pages():
    """The sequences that fit, in order, are served; nobody after the first that does not fit gets any."""
    t, ln, rf = i32([[0, -1, -1], [1, -1, -1], [2, -1, -1], [3, 4, -1]]), i32([4, 4, 4, 6]), i32([1, 1, 1, 1, 1, 0, 0])
    got, copies = bv.bv_pages_extend(t, ln, rf, 4, 8, i32([4, 8, 4, 2]))
    assert got.tolist() == [4, -1, -1, 2]                        # one page, two where one is left, none left, none needed
    assert ln.tolist() == [8, 4, 4, 8] and rf.tolist() == [1, 1, 1, 1, 1, 1, 0] and t.tolist()[0] == [0, 5, -1]
    assert (copies == -1).all()


def test_lengths_next_to_2_to_the_31():
    page, most = 1 << 20, 2**31 - 1024
    table = torch.zeros((3, 2048), dtype=torch.int32, device="cuda")
    lens = torch.tensor([most - 1, most, most + 1], dtype=torch.int32, device="cuda")
    refs = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    new, _ = bv.bv_pages_extend(table, lens, refs, page, 1)
    assert new.tolist() == [1, -1, -1] and lens.tolist() == [most, most, most + 1]
    bv.bv_pages_truncate(table, lens, refs, page, torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda"), 1)
    assert lens.tolist() == [most - 1, most - 1, most + 1] and refs.tolist() == [1, 0]


def test_a_table_that_names_a_free_page_keeps_it():
    """Such an entry is a fault of its own: compacting gives it no other page, whatever an earlier call left in the workspace."""
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        refs = (torch.rand(500, generator=g) < 0.4).int()
        before = torch.full((1, 500), -1, dtype=torch.int32)
        used = refs.nonzero().squeeze(1).int()
        before[0, :len(used)] = used
        table, lens = before.cuda(), i32([len(used)])
        bv.bv_pages_compact(table, lens, refs.cuda(), 1)               # leaves its moves in the workspace
        free = (refs == 0).nonzero().squeeze(1).int()
        wrong = torch.cat([used[:50], free[-100:]])[None].contiguous()
        cleared = refs.clone()
        cleared[used[50:]] = 0
        book = cp.Book(wrong, torch.tensor([150]), cleared, 1)
        moves, count = book.compact()
        table, lens = wrong.cuda(), i32([150])
        got_moves, got_count = bv.bv_pages_compact(table, lens, cleared.cuda(), 1)
        assert got_count.item() == count and got_moves.tolist() == moves and table.tolist() == book.table
        # pages that move now, and then come free while an entry still names them
        table = i32([used[50:].tolist()])
        bv.bv_pages_compact(table, i32([table.shape[1]]), cleared.cuda(), 1)
        assert table.tolist() == [used[50:].tolist()]


def test_shared_pages_are_replaced():
    t, ln, rf = i32([[0, 1, -1], [0, 1, -1], [0, 1, -1]]), i32([6, 6, 4]), i32([3, 3, 0, 0, 0])
    got, copies = bv.bv_pages_extend(t, ln, rf, 4, 1)
    # both that share the partly filled page get one of their own; the third, whose last token ends a page, a new one
    assert got.tolist() == [1, 1, 1] and copies.tolist() == [[1, 2], [1, 3], [-1, -1]]
    assert t.tolist() == [[0, 2, -1], [0, 3, -1], [0, 4, -1]] and rf.tolist() == [3, 1, 1, 1, 1]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,layout", [((9, 2, 16, 64), "heads"), ((9, 3, 5, 33), "heads"), ((9, 2, 16, 64), "tokens"), ((9, 1, 1, 8), "heads"), ((6, 8, 64, 128), "sliced")])
def test_copies(dtype, shape, layout):
    P, H, page, D = shape
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(dtype)                    # noqa: E731
    if layout == "tokens":
        k, v = rand(P, page, H, D).transpose(1, 2), rand(P, page, H, D).transpose(1, 2)
    elif layout == "sliced":
        k, v = rand(P, H, page, 2 * D)[..., :D], rand(P, 2 * H, page, D)[:, ::2]
    else:
        k, v = rand(P, H, page, D), rand(P, H, page, D)
    pairs = i32([[0, 5], [-1, -1], [1, 4], [2, P], [P, 3], [2, 2], [-1, 3], [2, 3]])
    for count, last in ((None, True), (i32([7]), False), (i32([99]), True), (i32([-1]), None)):
        a, b = k.clone(), v.clone()
        wa, wb = a.clone(), b.clone()
        for s, d in [] if last is None else [(0, 5), (1, 4)] + ([(2, 3)] if last else []):
            wa[d], wb[d] = a[s], b[s]
        kk, vv = torch.empty_strided(k.shape, k.stride(), dtype=dtype, device="cuda"), torch.empty_strided(v.shape, v.stride(), dtype=dtype, device="cuda")
        kk.copy_(k)
        vv.copy_(v)
        bv.bv_pages_copy(kk, vv, pairs, count)
        assert torch.equal(kk, wa) and torch.equal(vv, wb)


def test_bookkeeping_is_captured_and_replayed():
    t, ln, rf = i32([[0, -1, -1, -1], [1, -1, -1, -1]]), i32([3, 4]), i32([1, 1, 0, 0, 0, 0, 0, 0])
    book = cp.Book(t, ln, rf, 4)
    keep = i32([2, 1])
    bv.bv_pages_compact(t.clone(), ln.clone(), rf.clone(), 4)                                 # (the library is set up before any capture)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        new, _ = bv.bv_pages_extend(t, ln, rf, 4, 3, stream=s)
        bv.bv_pages_truncate(t, ln, rf, 4, keep, 3, new, stream=s)
        bv.bv_pages_compact(t, ln, rf, 4, stream=s)
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        got, _ = book.extend(3)
        book.truncate([2, 1], 3, got)
        book.compact()
        same(book, t, ln, rf)
