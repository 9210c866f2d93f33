"""The key-value cache that a speculative decoder keeps between verifications, as measurable cases.

A cache is two tensors of pages, ``k`` and ``v`` [pages, kv heads, page size, D], and for the sequences a table [B, table
width] of page numbers (token j of sequence b lies in page table[b, j // page size], row j % page size; -1: no page),
their lengths [B] and, for each page, how many table entries name it.  One iteration makes room for the block that is to be
scored (extend, which gives every sequence whose last page is shared a copy of its own), stores the block's keys and values
(append), lets its tokens attend to the cache (attend), and after the verification gives back what was not accepted
(truncate).  Sequences are forked into branches, and a pool with holes is compacted.  A case's ``op`` is one of

  attend    attention of the newest ``n`` tokens of each sequence over its pages: causal, ``Hq`` query heads on ``Hkv``
            key-value heads; with ``window`` > 0 a token sees the last ``window`` positions (itself among them) and the
            first ``sinks`` ones.  ``ragged``: sequence b brings only n_new[b] of the n tokens, the other rows stay as they are
  append    the keys and values of the newest ``n`` tokens into their pages
  branch    fork B sequences, extend the branches by ``n`` tokens, copy what extending them asks for, keep a part of each block
  compact   half of the sequences end, the others' pages move to the front of the pool, as many new ones are admitted

``L`` is the longest sequence, ``spare`` the pages that no sequence holds.
"""
import math

import torch

own = False

GOLDEN = 0.6180339887498949


def _case(name, op, B, n, Hq, Hkv, D, page, L, dtype="bf16", window=0, sinks=0, ragged=False, spare=64):
    c = dict(op=op, B=B, n=n, Hq=Hq, Hkv=Hkv, D=D, page=page, L=L, dtype=dtype, window=window, sinks=sinks,
             ragged=ragged, spare=spare)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a small draft model's step for one request: the smallest call, all latency
        _case("attend_1", "attend", 1, 1, 8, 8, 64, 16, 1000),
        # one request with a long context: the work of one sequence has to be split over the whole GPU
        _case("attend_long", "attend", 1, 1, 32, 8, 128, 64, 131072),
        # an ordinary batch that decodes token by token, sequences of all lengths
        _case("attend_64", "attend", 64, 1, 32, 8, 128, 16, 8192),
        # the scoring pass of a block of 8 drafted tokens: 72 query rows share every key
        _case("score_64", "attend", 64, 9, 64, 8, 128, 32, 16384),
        # 32-bit cache, sizes that are multiples of nothing, blocks of different lengths in one batch
        _case("score_odd_f32", "attend", 7, 5, 10, 2, 80, 24, 4001, dtype="f32", ragged=True),
        # a model with a sliding window and sinks: most of the cache is never read
        _case("window_128", "attend", 128, 1, 16, 4, 128, 16, 16384, window=1024, sinks=4),
        # the same for blocks, with an odd window that begins and ends inside pages
        _case("window_score_odd", "attend", 12, 6, 14, 2, 64, 48, 6000, window=333, sinks=5, ragged=True),
        # the block's keys and values of an ordinary batch
        _case("append_64", "append", 64, 9, 64, 8, 128, 32, 1500),
        # prompts of different lengths that enter the cache
        _case("append_prompts", "append", 16, 2048, 32, 8, 128, 64, 2048, ragged=True),
        # a few requests forked for a second draft each
        _case("branch_8", "branch", 8, 9, 8, 8, 64, 16, 1500, spare=512),
        # a full batch of them over a large pool with holes
        _case("branch_256", "branch", 256, 9, 8, 2, 64, 16, 2000, spare=20000),
        # half of a batch ends: the other half's pages move
        _case("compact_64", "compact", 64, 1, 32, 8, 128, 16, 2000, spare=4096),
    ]


KINDS = (("attend", 7), ("window", 3), ("append", 2), ("branch", 1), ("compact", 1))
LARGEST = 2.2e9          # bytes of a cache


def draw(rng):
    kind = rng.choices([k for k, _ in KINDS], [w for _, w in KINDS])[0]
    dtype = rng.choice(("bf16", "bf16", "bf16", "bf16", "f32"))
    D = rng.choice((64, 64, 128, 128, 128, 128, 80, 96))
    Hkv = rng.choice((1, 2, 4, 8))
    group = rng.choice((1, 2, 3, 4, 4, 5, 7, 8))
    page = rng.choice((16, 16, 32, 64, 128, 24, 48))
    token = 2 * Hkv * D * (4 if dtype == "f32" else 2)          # bytes of keys and values

    def spread(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))

    if kind in ("attend", "window"):
        B = spread(1, 192)
        L = spread(64, 65536)
        while B * L * token > LARGEST or B * L * Hkv * D > 3e8:      # (the plain form spreads the cache out in 32 bits)
            B, L = max(1, B // 2), max(64, L * 3 // 4)
        n = rng.choice((1, 1, 1, 3, 5, 6, 9, 9, 13, 17))
        while dtype == "f32" and n * group * B * L * Hkv > 1.5e8:
            n, group = max(1, n // 2), max(1, group // 2)
        window = spread(64, 4096) if kind == "window" else 0
        sinks = rng.choice((0, 1, 4, 4, 5, 16)) if kind == "window" else 0
        return _case(None, "attend", B, n, Hkv * group, Hkv, D, page, max(L, n), dtype, window, sinks, n > 1 and rng.random() < 0.3)
    if kind == "append":
        B, n = spread(1, 192), spread(1, 2048)
        while B * n * token > 1.3e8:
            B, n = max(1, B // 2), max(1, n * 3 // 4)
        return _case(None, "append", B, n, Hkv * group, Hkv, D, page, n + spread(1, 1000), dtype, ragged=rng.random() < 0.5)
    B = spread(2, 256)
    L = spread(64, 4000)
    while B * L * token > 6e8:
        B, L = max(2, B // 2), max(64, L * 3 // 4)
    if kind == "branch":
        return _case(None, "branch", B, rng.choice((1, 3, 5, 9, 17)), Hkv * group, Hkv, D, page, L, dtype, spare=spread(16, 8000) + 3 * B)
    return _case(None, "compact", B - B % 2, 1, Hkv * group, Hkv, D, page, L, dtype, spare=spread(16, 2000))


# ---- sizes that follow from a case -------------------------------------------------------------------------------------

def _lengths(case):
    """Sequence lengths between a sixteenth of the longest and the longest, evenly spread; never less than the block."""
    B, L, n = case["B"], case["L"], case["n"]
    floor = max(n, 1)
    return [max(floor, min(L, int(L * (1 / 16 + 15 / 16 * (1 - (i * GOLDEN) % 1.0))))) for i in range(B)]


def _n_new(case):
    """How many tokens each sequence brings: all n, or with ``ragged`` anything from none to all."""
    B, n = case["B"], case["n"]
    if not case["ragged"]:
        return [n] * B
    return [n if i == 0 else int((n + 1) * ((i * GOLDEN + 0.37) % 1.0)) for i in range(B)]


def _pages(tokens, page):
    return -(-tokens // page)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    B, n, Hq, Hkv, D, page = (case[k] for k in ("B", "n", "Hq", "Hkv", "D", "page"))
    lens, news = _lengths(case), _n_new(case)
    if case["op"] == "attend":
        tokens = pairs = entries = 0
        for L, m in zip(lens, news):
            if m == 0:
                continue
            first = L - m                                        # position of the block's first token
            if case["window"] > 0:
                lo = max(0, first - case["window"] + 1)
                sinks = min(case["sinks"], L)
                seen = L - lo + min(sinks, lo)
                for p in range(first, L):
                    low = max(0, p - case["window"] + 1)
                    pairs += p + 1 - low + min(sinks, low)
            else:
                seen = L
                pairs += m * (first + 1) + m * (m - 1) // 2
            tokens += seen
            entries += _pages(seen, page)
        return {"bytes": 2 * tokens * Hkv * D * es + 2 * sum(news) * Hq * D * es + 4 * entries + 8 * B, "flops": 4 * pairs * Hq * D}
    if case["op"] == "append":
        return {"bytes": 4 * sum(news) * Hkv * D * es + 4 * sum(_pages(m, page) for m in news) + 8 * B, "flops": 0}
    page_bytes = 2 * page * Hkv * D * es
    if case["op"] == "branch":
        shared = sum(1 for L in lens if L % page)                # branches whose last page is shared and not full
        held = sum(_pages(L, page) for L in lens)
        # the pages copied, the rows of the table read and written, the counts of the pages shared, the counts searched for free pages
        return {"bytes": 2 * shared * page_bytes + 16 * held + 4 * (held + case["spare"]) + 32 * B, "flops": 0}
    a, b = (sum(_pages(L, page) for L in lens[g::2]) for g in (0, 1))
    pool = a + b + case["spare"]
    return {"bytes": 2 * min(a, b) * page_bytes + 8 * pool + 16 * (a + b), "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _filled(shape, dtype, gen, scale=1.0):
    """Normal values, drawn in pieces: a large cache is not held in 32 bits besides."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn((part.numel(),), device="cuda", generator=gen).mul_(scale))
    return x


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    B, n, Hq, Hkv, D, page = (case[k] for k in ("B", "n", "Hq", "Hkv", "D", "page"))
    dtype, lens, news = _dtype(case), _lengths(case), _n_new(case)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")          # noqa: E731
    held = [_pages(x, page) for x in lens]
    rows = B
    if case["op"] == "branch":
        rows, width = 2 * B, _pages(max(lens) + n, page) + 1
    else:
        width = max(held)
    pool = sum(held) + case["spare"]
    order = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)  # sequences hold pages in no order, holes between them
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    column = torch.arange(width, device="cuda")[None, :]
    filled = column < i32(held)[:, None]
    table[:B][filled] = order[:sum(held)]
    lengths = i32(lens + [0] * (rows - B))
    refs = torch.zeros((pool,), dtype=torch.int32, device="cuda")
    refs[table[table >= 0].long()] = 1
    s = dict(case, k=_filled((pool, Hkv, page, D), dtype, gen), v=_filled((pool, Hkv, page, D), dtype, gen), table=table,
             lens=lengths, refs=refs)
    if case["op"] == "attend":
        # (queries of twice the keys' scale: a few keys in a thousand carry most of a row's weight)
        s["q"] = _filled((B, n, Hq, D), dtype, gen, 2.0)
        s["n_new"] = i32(news) if case["ragged"] else None
        s["out"] = torch.zeros((B, n, Hq, D), dtype=dtype, device="cuda")
    elif case["op"] == "append":
        s["k_new"], s["v_new"] = _filled((B, n, Hkv, D), dtype, gen), _filled((B, n, Hkv, D), dtype, gen)
        s["n_new"] = i32(news) if case["ragged"] else None
    elif case["op"] == "branch":
        s["src"], s["dst"] = i32(list(range(B))), i32(list(range(B, 2 * B)))
        s["n_new"] = i32([0] * B + [n] * B)
        # what a verification accepted of each branch's block
        s["keep"] = torch.randint(1, n + 1, (2 * B,), dtype=torch.int32, device="cuda", generator=gen)
    else:
        most = 2**31 - 1
        s["keep"] = [i32([0 if i % 2 == g else most for i in range(B)]) for g in (0, 1)]
        s["admit"] = [i32([x if i % 2 == g else 0 for i, x in enumerate(lens)]) for g in (0, 1)]
        s["longest"] = max(lens)
        s["turn"] = 0
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(s):
    op = s["op"]
    if own:
        return _own(s)
    if op == "attend":
        return _plain_attend(s)
    if op == "append":
        _plain_append(s)
        return s["k"], s["v"]
    if op == "branch":
        _plain_fork(s["table"], s["lens"], s["refs"], s["page"], s["src"], s["dst"])
        new, copies = _plain_extend(s["table"], s["lens"], s["refs"], s["page"], s["n"], s["n_new"])
        _plain_copy(s["k"], s["v"], copies)
        _plain_truncate(s["table"], s["lens"], s["refs"], s["page"], s["keep"], s["n"], new)
        return s["table"], s["lens"], s["refs"], new, copies, s["k"], s["v"]
    turn = s["turn"]
    s["turn"] = 1 - turn
    _plain_truncate(s["table"], s["lens"], s["refs"], s["page"], s["keep"][turn], 0, None)
    moves, count = _plain_compact(s["table"], s["lens"], s["refs"], s["page"])
    _plain_copy(s["k"], s["v"], moves)
    new, copies = _plain_extend(s["table"], s["lens"], s["refs"], s["page"], s["longest"], s["admit"][turn])
    return s["table"], s["lens"], s["refs"], moves, count, new, copies, s["k"], s["v"]


def _own(s):
    import paper_2403_10444_b200 as bv
    op = s["op"]
    if op == "attend":
        return bv.bv_cache_attend(s["q"], s["k"], s["v"], s["table"], s["lens"], n_new=s["n_new"], window=s["window"],
                                  sinks=s["sinks"], out=s["out"])
    if op == "append":
        bv.bv_cache_append(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["lens"], n_new=s["n_new"])
        return s["k"], s["v"]
    if op == "branch":
        bv.bv_pages_fork(s["table"], s["lens"], s["refs"], s["page"], s["src"], s["dst"])
        new, copies = bv.bv_pages_extend(s["table"], s["lens"], s["refs"], s["page"], s["n"], s["n_new"])
        bv.bv_pages_copy(s["k"], s["v"], copies)
        bv.bv_pages_truncate(s["table"], s["lens"], s["refs"], s["page"], s["keep"], s["n"], new)
        return s["table"], s["lens"], s["refs"], new, copies, s["k"], s["v"]
    turn = s["turn"]
    s["turn"] = 1 - turn
    bv.bv_pages_truncate(s["table"], s["lens"], s["refs"], s["page"], s["keep"][turn])
    moves, count = bv.bv_pages_compact(s["table"], s["lens"], s["refs"], s["page"])
    bv.bv_pages_copy(s["k"], s["v"], moves, count)
    new, copies = bv.bv_pages_extend(s["table"], s["lens"], s["refs"], s["page"], s["longest"], s["admit"][turn])
    return s["table"], s["lens"], s["refs"], moves, count, new, copies, s["k"], s["v"]


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _visible(s, positions):
    """[B, n, positions]: may token t of sequence b see position j?  And which of the n rows the sequence brings, [B, n]."""
    n, lens = s["n"], s["lens"].long()
    new = torch.full_like(lens, n) if s["n_new"] is None else s["n_new"].long()
    t = torch.arange(n, device=lens.device)
    at = (lens - new)[:, None] + t[None, :]                     # positions of the block's tokens
    j = torch.arange(positions, device=lens.device)
    see = j[None, None, :] <= at[:, :, None]
    if s["window"] > 0:
        see &= (j[None, None, :] > at[:, :, None] - s["window"]) | (j[None, None, :] < s["sinks"])
    return see, t[None, :] < new[:, None]


def _plain_attend(s):
    q, k, v, table = s["q"], s["k"], s["v"], s["table"]
    B, n, Hq, D = q.shape
    _, Hkv, page, _ = k.shape
    group, width = Hq // Hkv, table.shape[1]
    at = table.long().clamp_min(0)
    see, brought = _visible(s, width * page)
    # [B, Hkv, positions, D], each sequence's pages one after the other
    keys = k[at].transpose(1, 2).reshape(B, Hkv, width * page, D).float()
    rows = q.reshape(B, n, Hkv, group, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * group, D).float()
    score = torch.matmul(rows, keys.transpose(2, 3)).div_(math.sqrt(D))
    del keys
    mask = see[:, None, :, None, :].expand(B, 1, n, group, width * page).reshape(B, 1, n * group, width * page)
    score.masked_fill_(~mask, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    values = v[at].transpose(1, 2).reshape(B, Hkv, width * page, D).float()
    out = torch.matmul(score, values) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.reshape(B, Hkv, n, group, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D).to(q.dtype)
    return torch.where(brought[:, :, None, None], out, s["out"])


def _plain_append(s):
    k, page, n, lens = s["k"], s["page"], s["n"], s["lens"].long()
    new = torch.full_like(lens, n) if s["n_new"] is None else s["n_new"].long()
    t = torch.arange(n, device=lens.device)
    at = (lens - new)[:, None] + t[None, :]
    b, i = (t[None, :] < new[:, None]).nonzero(as_tuple=True)
    at = at[b, i]
    pages = s["table"].long()[b, at // page]
    k[pages, :, at % page] = s["k_new"][b, i]
    s["v"][pages, :, at % page] = s["v_new"][b, i]


def _held(lens, page):
    return (lens.long() + page - 1) // page


def _count(refs, pages, mask, by):
    """Adds ``by`` to the counts of the pages of a table that ``mask`` names."""
    refs.index_add_(0, pages.clamp(min=0).reshape(-1).long(), (mask.to(torch.int32) * by).reshape(-1))


def _plain_fork(table, lens, refs, page, src, dst):
    column = torch.arange(table.shape[1], device=table.device)[None, :]
    src, dst = src.long(), dst.long()
    taken, given = table[src], table[dst]
    _count(refs, taken, column < _held(lens[src], page)[:, None], 1)
    _count(refs, given, column < _held(lens[dst], page)[:, None], -1)
    table[dst] = torch.where(column < _held(lens[src], page)[:, None], taken, torch.full_like(taken, -1))
    lens[dst] = lens[src]


def _plain_extend(table, lens, refs, page, n, n_new):
    """Every sequence, in order, takes the lowest free pages; its last page, if shared and not full, is replaced first."""
    B, width = table.shape
    new = torch.full_like(lens, n) if n_new is None else n_new
    held = _held(lens, page)
    last = table.gather(1, (held - 1).clamp_min(0)[:, None])[:, 0]
    own_copy = (new > 0) & (lens % page > 0) & (refs[last.long().clamp_min(0)] > 1)
    need = (_held(lens + new, page) - held + own_copy).clamp_min(0)
    upto = need.cumsum(0)
    free = refs == 0
    served = ((upto <= free.sum()) | (need == 0)) & (lens.long() + new <= width * page) & (new >= 0)
    # free pages in order, by rank
    rank = torch.where(free, free.long().cumsum(0) - 1, refs.numel())
    by_rank = torch.zeros((refs.numel() + 1,), dtype=torch.long, device=table.device)
    by_rank.scatter_(0, rank, torch.arange(refs.numel(), device=table.device))
    column = torch.arange(width, device=table.device)[None, :]
    first = held - own_copy.long()
    takes = served[:, None] & (column >= first[:, None]) & (column < (first + need)[:, None])
    pages = by_rank[((upto - need)[:, None] + column - first[:, None]).clamp(0, refs.numel())]
    table.copy_(torch.where(takes, pages.to(torch.int32), table))
    _count(refs, table, takes, 1)
    own_copy &= served
    _count(refs, last, own_copy, -1)
    replaced = table.gather(1, (held - 1).clamp_min(0)[:, None])[:, 0]
    none = torch.full_like(last, -1)
    lens.add_(torch.where(served, new, torch.zeros_like(new)))
    return torch.where(served, new, none), torch.stack([torch.where(own_copy, last, none), torch.where(own_copy, replaced, none)], 1)


def _plain_truncate(table, lens, refs, page, keep, n, n_new):
    """Of the n newest tokens (n = 0: of all) only the first ``keep`` stay; pages that no longer hold any are given back."""
    new = lens if n == 0 else torch.minimum((torch.full_like(lens, n) if n_new is None else n_new).clamp_min(0), lens)
    length = lens - new + torch.minimum(keep.clamp_min(0), new)
    column = torch.arange(table.shape[1], device=table.device)[None, :]
    gone = (column >= _held(length, page)[:, None]) & (column < _held(lens, page)[:, None])
    _count(refs, table, gone, -1)
    table.masked_fill_(gone, -1)
    lens.copy_(length)


def _plain_compact(table, lens, refs, page):
    """The pages in use beyond the number of pages in use move, in order, into the free pages before it, in order."""
    P = refs.numel()
    used = refs > 0
    live = used.sum()
    at = torch.arange(P, device=table.device)
    source, hole = used & (at >= live), ~used & (at < live)
    count = source.sum()
    moves = torch.full((P // 2 + 1, 2), -1, dtype=torch.int32, device=table.device)
    for column, which in ((0, source), (1, hole)):
        rank = torch.where(which, which.long().cumsum(0) - 1, P // 2)
        moves[:, column].scatter_(0, rank, at.to(torch.int32))
    moves = moves[:P // 2]
    moves[torch.arange(P // 2, device=table.device) >= count] = -1
    to = torch.cat([at, at[:1]])
    valid = moves[:, 0] >= 0
    to.scatter_(0, torch.where(valid, moves[:, 0].long(), P), torch.where(valid, moves[:, 1].long(), 0))
    named = torch.arange(table.shape[1], device=table.device)[None, :] < _held(lens, page)[:, None]
    table.copy_(torch.where(named, to[table.long().clamp_min(0)].to(torch.int32), table))
    counts = torch.zeros((P + 1,), dtype=torch.int32, device=table.device)
    counts.scatter_(0, torch.where(used, to[:P], P), refs)
    refs.copy_(counts[:P])
    return moves, count.to(torch.int32).reshape(1)


def _plain_copy(k, v, pairs):
    pairs = pairs[pairs[:, 0] >= 0].long()
    k[pairs[:, 1]] = k[pairs[:, 0]]
    v[pairs[:, 1]] = v[pairs[:, 0]]


# ---- 64 bits -----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    """The attention in 64 bits, sequence by sequence from the definition; the other operators move what they are given."""
    if case["op"] != "attend":
        return None
    s = prepare(case, seed)
    q, k, v = s["q"], s["k"], s["v"]
    B, n, Hq, D = q.shape
    Hkv, page = k.shape[1], k.shape[2]
    out = torch.zeros((B, n, Hq, D), dtype=torch.float64, device=q.device)
    for b, (L, m) in enumerate(zip(_lengths(case), _n_new(case))):
        if m == 0:
            continue
        pages = s["table"][b, :_pages(L, page)].long()
        keys, values = (x[pages].permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :L].double() for x in (k, v))
        for t in range(m):
            p = L - m + t
            seen = torch.arange(p + 1, device=q.device)
            if case["window"] > 0:
                seen = seen[(seen > p - case["window"]) | (seen < case["sinks"])]
            rows = q[b, t].double().reshape(Hkv, Hq // Hkv, D)
            # (all of a long sequence is visible: no copy of it per token)
            some = keys[:, :p + 1] if seen.numel() == p + 1 else keys[:, seen]
            weight = torch.softmax(torch.einsum("hgd,hjd->hgj", rows, some) * D ** -0.5, dim=-1)
            some = values[:, :p + 1] if seen.numel() == p + 1 else values[:, seen]
            out[b, t] = torch.einsum("hgj,hjd->hgd", weight, some).reshape(Hq, D)
    return out
