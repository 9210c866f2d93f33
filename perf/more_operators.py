"""What a speculative decoder does with a prompt and with its rows of logits, as measurable cases.

A case's ``op`` is one of

  rope      the queries and keys of the newest tokens are rotated by the angles of their positions, and keys and values go into the
            pages of a cache (k, v [pages, kv heads, page size, D]; token j of sequence b lies in page table[b, j // page size]).
            ``rot`` of a head's D elements are rotated, in pairs (i, i + rot / 2) or, ``interleaved``, (2 i, 2 i + 1); pair i turns by
            position times freq[i] (64 bits), and what is rotated is scaled by ``mscale``.  ``packed``: the tokens of all
            sequences lie one after the other and ``offsets`` says where each sequence's begin; else they are [B, n, ...], and with
            ``ragged`` sequence b brings only n_new[b] of the n.  ``start``: how long the longest sequence was before
  prompt    causal attention of whole prompts of different lengths that lie one after the other: q [tokens, Hq, D] on k, v [tokens,
            Hkv, D], sequence b from offsets[b] to offsets[b + 1]; with ``window`` > 0 a token sees the last ``window`` positions (itself among
            them) and the first ``sinks`` ones.  ``tail`` rows behind the last sequence stay as they are
  sample    rows of logits at a temperature, cut to the ``top_k`` largest, of those to the smallest set with ``top_p`` of their mass, and to
            tokens at least ``min_p`` times as likely as the likeliest; a token drawn from what is left by inverse CDF in the order of
            the vocabulary, the log of what its weights add up to, and the rows with the others at -inf, as a verification takes them
  filter    the same without the drawing: the target's rows

``mixed``: every row has parameters of its own.  Equal logits count in the order of the vocabulary.
"""
import math

import torch

own = False

GOLDEN = 0.6180339887498949


def _rope(name, B, n, Hq, Hkv, D, page, start, rot, dtype="bf16", interleaved=False, packed=False, ragged=False, mscale=1.0, base=10000.0):
    c = dict(op="rope", B=B, n=n, Hq=Hq, Hkv=Hkv, D=D, page=page, start=start, rot=rot, dtype=dtype, interleaved=interleaved, packed=packed,
             ragged=ragged, mscale=mscale, base=base)
    return dict(c, name=name) if name else c


def _prompt(name, B, L, Hq, Hkv, D, dtype="bf16", window=0, sinks=0, tail=0):
    c = dict(op="prompt", B=B, L=L, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, window=window, sinks=sinks, tail=tail)
    return dict(c, name=name) if name else c


def _rows(name, op, rows, V, dtype="bf16", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, zipf=True):
    c = dict(op=op, rows=rows, V=V, dtype=dtype, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, mixed=mixed, zipf=zipf)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the block of 9 tokens of an ordinary batch, scored by a target with rotated heads
        _rope("rope_64", 64, 9, 64, 8, 128, 32, 1500, 128),
        # prompts that enter the cache, a context stretched to eight times what the frequencies were made for
        _rope("rope_prompts", 16, 2048, 32, 8, 128, 64, 0, 128, packed=True, ragged=True, mscale=1.2079, base=500000.0),
        # a 32-bit model of which a part of the head turns, pairs side by side, far positions, blocks of different lengths
        _rope("rope_odd_f32", 7, 5, 10, 2, 80, 24, 130000, 36, dtype="f32", interleaved=True, ragged=True),
        # a short question to a small model: the smallest call, all latency
        _prompt("prompt_1", 1, 45, 8, 8, 64),
        # prompts of an ordinary batch
        _prompt("prompt_16", 16, 2048, 32, 8, 128),
        # one long document: all products
        _prompt("prompt_long", 1, 32768, 32, 8, 128),
        # a model with a sliding window and sinks
        _prompt("prompt_window", 8, 8192, 16, 4, 64, window=1024, sinks=4, tail=3),
        # 32 bits, sizes that are multiples of nothing
        _prompt("prompt_odd_f32", 7, 701, 10, 2, 80, dtype="f32", tail=5),
        # one request's drafting step with the usual settings
        _rows("sample_1", "sample", 1, 32000, temperature=0.7, top_k=50, top_p=0.95),
        # a batch's drafting step, nucleus of the whole vocabulary
        _rows("sample_64", "sample", 64, 128256, temperature=0.8, top_p=0.9),
        # a batch of requests with settings of their own, 32 bits, rows that are no whole vectors
        _rows("sample_odd_f32", "sample", 37, 50257, dtype="f32", mixed=True),
        # the target's rows of a batch of blocks of 9
        _rows("filter_576", "filter", 576, 128256, temperature=0.8, top_k=1000, top_p=0.95, min_p=0.01),
    ]


def draw(rng):
    kind = rng.choice(("rope", "rope", "prompt", "prompt", "prompt", "window", "rows", "rows", "rows"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))

    def spread(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))

    if kind == "rows":
        rows, V = spread(1, 576), rng.choice((spread(300, 256000), 32000, 50257, 128256, 152064))
        while rows * V > (37000000 if dtype == "f32" else 74000000):
            rows = max(1, rows // 2)
        return _rows(None, rng.choice(("sample", "sample", "filter")), rows, V, dtype, rng.choice((0.5, 0.7, 0.8, 1.0, 1.3)), rng.choice((0, 0, 1, 20, 50, 200, 1000)),
                     rng.choice((1.0, 0.5, 0.8, 0.9, 0.95, 0.99)), rng.choice((0.0, 0.0, 0.01, 0.05, 0.1)), rng.random() < 0.3, rng.random() < 0.7)
    D = rng.choice((64, 64, 128, 128, 128, 80, 96))
    Hkv = rng.choice((1, 2, 4, 8))
    Hq = Hkv * rng.choice((1, 2, 3, 4, 4, 5, 7, 8))
    if kind == "rope":
        packed = rng.random() < 0.4
        B, n = spread(1, 192), spread(1, 2048) if packed else rng.choice((1, 1, 3, 5, 9, 9, 17))
        start = 0 if packed else spread(1, 100000)
        es = 4 if dtype == "f32" else 2
        # (the tokens that move, and pools that are made anew for every input)
        while B * n * (Hq + 2 * Hkv) * D * es > 2.6e8 or B * (n + start) * 2 * Hkv * D * es > 1.5e9:
            B, n, start = max(1, B // 2), max(1, n * 3 // 4), start * 3 // 4
        rot = rng.choice((D, D, D, D // 2, D // 4))
        return _rope(None, B, n, Hq, Hkv, D, rng.choice((16, 16, 32, 64, 24)), start, rot, dtype, rng.random() < 0.4, packed, n > 1 and rng.random() < 0.5,
                     rng.choice((1.0, 1.0, 1.1, 1.2079)), rng.choice((10000.0, 500000.0, 1000000.0)))
    B, L = spread(1, 96), spread(1, 32768)
    # (32 bits: the products of the largest 32-bit case, not of the largest)
    while B * L > 131072 or B * L * L * Hq * D > (1.0e11 if dtype == "f32" else 4.3e12):
        B, L = max(1, B // 2), max(1, L * 3 // 4)
    window = spread(16, 4096) if kind == "window" else 0
    return _prompt(None, B, L, Hq, Hkv, D, dtype, window, rng.choice((0, 1, 4, 16)) if window else 0, rng.choice((0, 0, 5)))


# ---- sizes that follow from a case -------------------------------------------------------------------------------------

def _spread(B, L, ragged=True):
    """B lengths between a sixteenth of L and L, evenly spread, the first of them L."""
    return [L if i == 0 or not ragged else max(1, int(L * (1 / 16 + 15 / 16 * (1 - (i * GOLDEN) % 1.0)))) for i in range(B)]


def _brings(case):
    """How many tokens each sequence of a ``rope`` case brings."""
    if case["packed"]:
        return _spread(case["B"], case["n"], case["ragged"])
    n = case["n"]
    return [n if i == 0 or not case["ragged"] else int((n + 1) * ((i * GOLDEN + 0.37) % 1.0)) for i in range(case["B"])]


def _before(case):
    """How long the sequences of a ``rope`` case were before."""
    return _spread(case["B"], case["start"]) if case["start"] else [0] * case["B"]


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _settings(case):
    """(temperature, top_k, top_p, min_p) of each row."""
    if not case["mixed"]:
        return [(case["temperature"], case["top_k"], case["top_p"], case["min_p"])] * case["rows"]
    some = ((1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (0.6, 20, 0.95, 0.0), (1.2, 200, 0.9, 0.02), (1.0, 1, 1.0, 0.0))
    return [some[i % len(some)] for i in range(case["rows"])]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("sample", "filter"):
        # the rows in, the rows out
        n = case["rows"] * case["V"]
        return {"bytes": 2 * n * es + (12 * case["rows"] if case["op"] == "sample" else 0), "flops": 2 * n}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "rope":
        m = sum(_brings(case))
        # queries in and out, keys and values in and into their pages; packed: the turned keys beside, for the prompts' attention
        heads = 2 * Hq + 4 * Hkv + (Hkv if case["packed"] else 0)
        return {"bytes": m * heads * D * es + 4 * case["rot"] + 12 * case["B"], "flops": 3 * m * (Hq + Hkv) * case["rot"]}
    lens = _spread(case["B"], case["L"])
    pairs = 0
    for L in lens:
        w, s = case["window"], case["sinks"]
        if w == 0 or w >= L:
            pairs += L * (L + 1) // 2
        else:
            pairs += w * (w + 1) // 2 + (L - w) * w
            # sinks that lie before the windows: positions p from w on see min(s, p - w + 1) of them
            full = max(0, L - w - max(0, s - 1))
            pairs += full * s + sum(min(s, x) for x in range(1, L - w - full + 1))
    return {"bytes": sum(lens) * (2 * Hq + 2 * Hkv) * D * es + 4 * (case["B"] + 1), "flops": 4 * pairs * Hq * D}


# ---- inputs ------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _dtype(case)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")                                # noqa: E731
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=gen).to(dtype)               # noqa: E731
    offsets = lambda lens: i32([sum(lens[:i]) for i in range(len(lens) + 1)])                        # noqa: E731
    s = dict(case)
    if case["op"] in ("sample", "filter"):
        rows, V = case["rows"], case["V"]
        z = torch.empty((rows, V), dtype=dtype, device="cuda")
        fall = -1.1 * torch.log(torch.arange(1, V + 1, dtype=torch.float32, device="cuda"))
        for i in range(0, rows, 64):
            part = z[i:i + 64]
            x = torch.randn(part.shape, device="cuda", generator=gen)
            if case["zipf"]:
                # (a rank law under a random order of each row, and noise)
                order = torch.rand(part.shape, device="cuda", generator=gen).argsort(1)
                part.copy_(x.mul_(0.3).add_(fall[order]))
            else:
                part.copy_(x.mul_(3.0))
        s.update(logits=z, uniforms=torch.rand((rows,), device="cuda", generator=gen), filtered=torch.empty_like(z))
        if case["mixed"]:
            t, k, p, m = zip(*_settings(case))
            f32 = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")                      # noqa: E731
            s.update(temperature=f32(t), top_k=i32(k), top_p=f32(p), min_p=f32(m))
        return s
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "prompt":
        lens = _spread(case["B"], case["L"])
        T = sum(lens) + case["tail"]
        # (queries of twice the keys' scale: a few keys in a thousand carry most of a row's weight)
        s.update(q=normal(T, Hq, D).mul_(2), k=normal(T, Hkv, D), v=normal(T, Hkv, D), offsets=offsets(lens), out=torch.zeros((T, Hq, D), dtype=dtype, device="cuda"))
        return s
    B, n, page, news, before = case["B"], case["n"], case["page"], _brings(case), _before(case)
    lens = [x + m for x, m in zip(before, news)]
    held = [-(-x // page) for x in lens]
    pool = sum(held) + 64
    table = torch.full((B, max(held) + 1), -1, dtype=torch.int32, device="cuda")
    column = torch.arange(table.shape[1], device="cuda")[None, :]
    # (sequences hold pages in no order)
    table[column < i32(held)[:, None]] = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)[:sum(held)]
    shape = (sum(news),) if case["packed"] else (B, n)
    half = case["rot"] // 2
    freq = torch.arange(half, dtype=torch.float64, device="cuda").mul_(-2.0 / case["rot"] * math.log(case["base"])).exp_()
    if case["mscale"] != 1.0:
        freq[half // 2:] /= 8.0                    # (a stretched context: the slow pairs turn an eighth as fast)
    # q, k and v as one projection leaves them
    qkv = normal(*shape, Hq + 2 * Hkv, D)
    q, k_new, v_new = qkv.split([Hq, Hkv, Hkv], dim=-2)
    s.update(q=q, k_new=k_new, v_new=v_new, k=torch.zeros((pool, Hkv, page, D), dtype=dtype, device="cuda"),
             v=torch.zeros((pool, Hkv, page, D), dtype=dtype, device="cuda"), table=table, lens=i32(lens), freq=freq,
             n_new=i32(news) if case["ragged"] and not case["packed"] else None, offsets=offsets(news) if case["packed"] else None,
             out_q=torch.zeros((*shape, Hq, D), dtype=dtype, device="cuda"), out_k=torch.zeros((*shape, Hkv, D), dtype=dtype, device="cuda") if case["packed"] else None)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(s):
    op = s["op"]
    if own:
        return _own(s)
    if op == "rope":
        return _plain_rope(s)
    if op == "prompt":
        return _plain_prompt(s)
    return _plain_rows(s)


def _own(s):
    import paper_2403_10444_b200 as bv
    op = s["op"]
    if op == "rope":
        bv.bv_cache_append_rotary(s["q"], s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["lens"], s["freq"], n_new=s["n_new"], offsets=s["offsets"],
                                  interleaved=s["interleaved"], mscale=s["mscale"], out_q=s["out_q"], out_k=s["out_k"])
        return (s["out_q"], s["k"], s["v"]) if s["out_k"] is None else (s["out_q"], s["k"], s["v"], s["out_k"])
    if op == "prompt":
        return bv.bv_prompt_attend(s["q"], s["k"], s["v"], s["offsets"], window=s["window"], sinks=s["sinks"], out=s["out"])
    settings = dict(temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    if op == "filter":
        return bv.bv_filter_logits(s["logits"], out=s["filtered"], **settings)
    tokens, lse = bv.bv_sample_filtered(s["logits"], s["uniforms"], out_logits=s["filtered"], **settings)
    return tokens, lse, s["filtered"]


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _places(s):
    """(index of the sequence, position, which rows count) of each new token, as a list of all or [B, n]."""
    lens = s["lens"].long()
    if s["packed"]:
        off = s["offsets"].long()
        r = torch.arange(s["q"].shape[0], device=lens.device)
        b = torch.searchsorted(off, r, right=True) - 1
        return b, lens[b] - off[b + 1] + r, torch.ones_like(b, dtype=torch.bool)
    n = s["n"]
    new = torch.full_like(lens, n) if s["n_new"] is None else s["n_new"].long()
    t = torch.arange(n, device=lens.device)
    return torch.arange(lens.shape[0], device=lens.device)[:, None].expand(-1, n), (lens - new)[:, None] + t[None, :], t[None, :] < new[:, None]


def _turned(x, cos, sin, rot, interleaved):
    """x [..., heads, D] with its first ``rot`` elements turned."""
    y = x[..., :rot].float()
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else y.chunk(2, dim=-1)
    c, d = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([c, d], dim=-1).flatten(-2) if interleaved else torch.cat([c, d], dim=-1)
    return torch.cat([y.to(x.dtype), x[..., rot:]], dim=-1)


def _plain_rope(s):
    b, at, counts = _places(s)
    angle = at[..., None].double() * s["freq"]
    cos, sin = ((f * s["mscale"]).float()[..., None, :] for f in (angle.cos(), angle.sin()))
    q = _turned(s["q"], cos, sin, s["rot"], s["interleaved"])
    k = _turned(s["k_new"], cos, sin, s["rot"], s["interleaved"])
    s["out_q"][counts] = q[counts]
    page = s["page"]
    b, at = b[counts], at[counts]
    pages = s["table"].long()[b, at // page]
    s["k"][pages, :, at % page] = k[counts]
    s["v"][pages, :, at % page] = s["v_new"][counts]
    if s["out_k"] is None:
        return s["out_q"], s["k"], s["v"]
    s["out_k"].copy_(k)
    return s["out_q"], s["k"], s["v"], s["out_k"]


def _plain_prompt(s):
    q, k, v, out = s["q"], s["k"], s["v"], s["out"]
    Hq, D, Hkv = q.shape[1], q.shape[2], k.shape[1]
    first = 0
    # (a sequence after the other, a key-value head after the other: the scores of all do not fit)
    for L in _spread(s["B"], s["L"]):
        j = torch.arange(L, device=q.device)
        hidden = j[None, :] > j[:, None]
        if s["window"] > 0:
            hidden |= (j[None, :] <= j[:, None] - s["window"]) & (j[None, :] >= s["sinks"])
        rows, keys, values = (x[first:first + L].float() for x in (q, k, v))
        rows = rows.reshape(L, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3)
        for h in range(Hkv):
            score = torch.matmul(rows[h], keys[:, h].t()).div_(math.sqrt(D)).masked_fill_(hidden, -math.inf)
            score = score.sub_(score.amax(-1, keepdim=True)).exp_()
            total = score.sum(-1, keepdim=True)
            o = torch.matmul(score, values[:, h]).div_(total)
            out[first:first + L].view(L, Hkv, Hq // Hkv, D)[:, h] = o.permute(1, 0, 2).to(out.dtype)
        first += L
    return out


def _plain_rows(s):
    z = s["logits"]
    rows, V = z.shape
    each = lambda x: x[:, None] if s["mixed"] else x                                                 # noqa: E731
    one = lambda x: torch.tensor(x, dtype=torch.float32, device=z.device).double()                   # noqa: E731
    number = lambda x: x[:, None].double() if s["mixed"] else one(x)                                 # noqa: E731
    temperature, top_p, min_p, top_k = number(s["temperature"]), number(s["top_p"]), number(s["min_p"]), each(s["top_k"])
    # (sums of a whole vocabulary, next to whose borders a token is in or out: 64 bits)
    ordered, order = z.sort(dim=1, descending=True, stable=True)
    far = (ordered.double() - ordered[:, :1].double()) / temperature
    weight = far.exp()
    rank = torch.arange(V, device=z.device)[None, :]
    top_k = torch.as_tensor(top_k, device=z.device)
    keep = (rank < top_k) | (top_k <= 0)
    weight = torch.where(keep, weight, 0.0)
    upto = weight.cumsum(1)
    keep = keep & ((upto - weight < top_p * upto[:, -1:]) | (top_p >= 1) | (rank == 0)) & ((far >= min_p.log()) | (min_p <= 0))
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    filtered = torch.where(kept, z, torch.full_like(z, -math.inf))
    s["filtered"].copy_(filtered)
    if s["op"] == "filter":
        return s["filtered"]
    weight = torch.zeros_like(weight).scatter_(1, order, torch.where(keep, weight, 0.0))
    upto = weight.cumsum(1)
    total = upto[:, -1:]
    tokens = ((upto > s["uniforms"][:, None].double() * total) & (weight > 0)).to(torch.int32).argmax(1).to(torch.int32)
    lse = (ordered[:, 0].double() / (temperature[:, 0] if s["mixed"] else temperature) + total[:, 0].log()).float()
    return tokens, lse, s["filtered"]


# ---- 64 bits -----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "prompt": _exact_prompt}.get(case["op"], _exact_rows)(case, s)


def _exact_rope(case, s):
    """Sequence by sequence, pairs as complex numbers."""
    rot, Hq, page = case["rot"], case["Hq"], case["page"]
    half = rot // 2
    i = torch.arange(half, device="cuda")
    one, two = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
    out = {name: torch.zeros(s[name].shape, dtype=torch.float64, device="cuda") for name in ("out_q", "k", "v")}
    out_k = torch.zeros(s["out_k"].shape, dtype=torch.float64, device="cuda") if case["packed"] else None
    first = 0
    for b, (m, L) in enumerate(zip(_brings(case), _before(case))):
        at = torch.arange(L, L + m, dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full((m, half), float(case["mscale"]), dtype=torch.float64, device="cuda"), at[:, None] * s["freq"][None, :])
        here = (slice(first, first + m),) if case["packed"] else (b, slice(0, m))

        def turned(x):
            x = x.double().clone()
            z = torch.complex(x[..., one], x[..., two]) * turn[:, None, :]
            x[..., one], x[..., two] = z.real, z.imag
            return x

        out["out_q"][here] = turned(s["q"][here])
        k = turned(s["k_new"][here])
        if case["packed"]:
            out_k[here] = k
        pages, rows = s["table"][b].long()[at.long() // page], at.long() % page
        out["k"][pages, :, rows] = k
        out["v"][pages, :, rows] = s["v_new"][here].double()
        first += m
    return (out["out_q"], out["k"], out["v"], out_k) if case["packed"] else (out["out_q"], out["k"], out["v"])


def _exact_prompt(case, s):
    """Some hundred rows of one sequence and head at a time."""
    q, k, v = s["q"], s["k"], s["v"]
    Hq, D, Hkv = q.shape[1], q.shape[2], k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    first = 0
    for L in _spread(case["B"], case["L"]):
        for h in range(Hkv):
            keys, values = k[first:first + L, h].double(), v[first:first + L, h].double()
            mine = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            step = max(64, (1 << 25) // L)
            for t in range(0, L, step):
                end = min(L, t + step)
                p, j = torch.arange(t, end, device=q.device)[:, None], torch.arange(end, device=q.device)[None, :]
                see = j <= p
                if case["window"] > 0:
                    see &= (p - j < case["window"]) | (j < case["sinks"])
                score = torch.einsum("thd,jd->htj", q[first + t:first + end, mine].double(), keys[:end]) * D ** -0.5
                weight = torch.softmax(torch.where(see, score, -math.inf), dim=-1)
                out[first + t:first + end, mine] = torch.einsum("htj,jd->thd", weight, values[:end])
        first += L
    return out


def _exact_rows(case, s):
    """Row by row over the distinct values of its logits, largest first: how many of each are in."""
    tokens, lses, filtered = [], [], torch.full(s["logits"].shape, -math.inf, dtype=torch.float64, device="cuda")
    as_kept = lambda x: float(torch.tensor(x, dtype=torch.float32))                                  # noqa: E731
    for r, (T, k, p, m) in enumerate(_settings(case)):
        T, p, m = as_kept(T), as_kept(p), as_kept(m)
        z = s["logits"][r].double()
        value, which, count = torch.unique(z, return_inverse=True, return_counts=True)
        value, count = value.flip(0), count.flip(0)
        which = value.numel() - 1 - which
        each = ((value - value[0]) / T).exp()
        ahead = count.cumsum(0) - count
        some = count if k <= 0 else (k - ahead).clamp_min(0).minimum(count)
        mass = each * some
        before = mass.cumsum(0) - mass
        if p < 1:
            # of a value the i-th is in if the mass before it, that of larger ones and i of its own, is below the border
            i = torch.ceil((p * mass.sum() - before) / each).clamp(min=0)
            i[0] = i[0].clamp_min(1)
            some = torch.where(i < some, i.nan_to_num(0.0), some.double()).long()
        if m > 0:
            some = torch.where((value - value[0]) / T >= math.log(m), some, 0)
        # the lowest indices of a value come first
        by_value = which.sort(stable=True).indices
        place = torch.empty_like(which)
        place[by_value] = torch.arange(z.numel(), device=z.device) - ahead[which[by_value]]
        kept = place < some[which]
        filtered[r] = torch.where(kept, z, -math.inf)
        if case["op"] == "sample":
            w = torch.where(kept, ((z - value[0]) / T).exp(), 0.0)
            total = (each * some).sum()
            tokens.append(int(((w.cumsum(0) > s["uniforms"][r].double() * total) & (w > 0)).to(torch.int32).argmax()))
            lses.append(float(value[0]) / T + math.log(float(total)))
    if case["op"] == "filter":
        return filtered
    return torch.tensor(tokens, dtype=torch.int32, device="cuda"), torch.tensor(lses, dtype=torch.float64, device="cuda"), filtered
