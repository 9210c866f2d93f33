"""The decoding loop on the paged cache (cached.py): the tokens of a loop that keeps no cache and forms every logit anew from the whole
context in 64 bits, the caches' bookkeeping, replays, and the branches that forks make."""
import pytest
import torch

import cache_plain as cp
from paper_2403_10444_b200 import cached, specdec, workloads as wl
import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu


def dense_logits(w, tokens, window, sinks):
    """Logits after every token of one sequence, in float64: [L, V]."""
    x = w["embed"][tokens.long()].double()
    L, H, K, D = x.shape[0], w["heads"], w["kv_heads"], w["head_dim"]
    j = torch.arange(L, device=x.device)
    see = j[None, :] <= j[:, None]
    if window:
        see &= (j[None, :] > j[:, None] - window) | (j[None, :] < sinks)
    for layer in w["layers"]:
        qkv = (x @ layer["qkv"].double()).view(L, H + 2 * K, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + K].repeat_interleave(H // K, 1), qkv[:, H + K:].repeat_interleave(H // K, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) * D ** -0.5
        p = torch.softmax(s.masked_fill(~see, float("-inf")), -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(L, H * D) @ layer["out"].double()
    return x @ w["unembed"].double()


def plain_loop(tw, dw, prompts, lens, ud, uv, gamma, T, algo, window, sinks):
    """Algorithm 3 with no cache: the contexts as lists, every row of logits formed from the whole context in 64 bits and rounded to the
    loop's 32."""
    B = prompts.shape[0]
    ctx = [prompts[b, :lens[b]].tolist() for b in range(B)]
    start = [len(c) for c in ctx]
    dev = prompts.device
    last = lambda w, toks, n: torch.stack([dense_logits(w, torch.tensor(t, device=dev), window, sinks)[-n:] for t in toks]).float()      # noqa: E731
    for it in range(ud.shape[0]):
        toks = [list(c) for c in ctx]
        rows, lse = [], []
        for i in range(gamma):
            z = last(dw, toks, 1)[:, 0].contiguous()
            tok, l = bv.bv_sample_draft(z, ud[it, i].contiguous(), T)
            rows.append(z)
            lse.append(l)
            for t, x in zip(toks, tok.tolist()):
                t.append(x)
        drafted = torch.tensor([t[-gamma:] for t in toks], dtype=torch.int32, device=dev)
        target, draft = last(tw, toks, gamma + 1).contiguous(), torch.stack(rows, 1).contiguous()
        given = (torch.stack(lse, 1).contiguous(),) if algo.endswith("lse") else ()
        fn = {"block_lse": bv.bv_verify_lse, "token_lse": bv.tv_verify_lse, "block": bv.bv_verify, "token": bv.tv_verify}[algo]
        out, n = fn(target, draft, drafted, uv[it].contiguous(), *given, T)
        for c, row, k in zip(ctx, out.tolist(), n.tolist()):
            assert k >= 1
            c += row[:k]
    return [c[s:] for c, s in zip(ctx, start)]


def setup(dtype="f32", V=512, B=5, L=40, N=5, gamma=3, seed=0, heads=4, kv_heads=2, head_dim=32, page=16, window=0, sinks=0, noise=0.05):
    tw, dw = wl.attention_models(V, dtype, seed, 2, heads, kv_heads, head_dim, noise, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    prompts = torch.randint(V, (B, L), dtype=torch.int32, device="cuda", generator=g)
    lens = torch.randint(1, L + 1, (B,), dtype=torch.int32, device="cuda", generator=g)
    lens[0], lens[1] = 1, L
    ud, uv = wl.loop_uniforms(N, B, gamma, seed + 1, "cuda")
    make = lambda: [cached.Decoder(w, B, L + N * (gamma + 1), page, window, sinks) for w in (tw, dw)]       # noqa: E731
    return tw, dw, prompts, lens, ud, uv, make


@pytest.mark.parametrize("algo", specdec.ALGOS)
@pytest.mark.parametrize("window,sinks,page", [(0, 0, 16), (9, 2, 5)])
def test_the_loop_is_that_without_a_cache(algo, window, sinks, page):
    tw, dw, prompts, lens, ud, uv, make = setup(window=window, sinks=sinks, page=page)
    res = cached.run(*make(), prompts, lens, ud, uv, 3, 0.9, algo)
    want = plain_loop(tw, dw, prompts, lens, ud, uv, 3, 0.9, algo, window, sinks)
    for b, toks in enumerate(want):
        assert res["tokens"][b, :len(toks)].tolist() == toks and int(res["lengths"][b]) == len(toks)
        assert (res["tokens"][b, len(toks):] == -1).all()
    assert res["tau"].float().mean() > 0.5           # (drafts are accepted, and rejected, so the caches are cut back)
    assert (res["tau"] < 3).any()


@pytest.mark.parametrize("dtype,head_dim", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_the_caches_afterwards(dtype, head_dim):
    tw, dw, prompts, lens, ud, uv, make = setup(dtype, head_dim=head_dim, B=7, L=100, N=6, gamma=4, heads=8)
    models = make()
    res = cached.run(*models, prompts, lens, ud, uv, 4, 1.0)
    for m in models:
        c = m.cache
        # all tokens but the last emitted one are in the cache, on pages of their own
        assert torch.equal(c.lens.long(), lens.long() - 1 + res["lengths"])
        named = c.table[c.table >= 0]
        assert torch.equal(torch.bincount(named.long(), minlength=c.refs.numel()).int(), c.refs) and c.refs.max() == 1
        assert named.numel() == sum(cp.ceil_div(x, c.page_size) for x in c.lens.tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replays_of_a_captured_iteration_give_the_same_tokens(dtype):
    tw, dw, prompts, lens, ud, uv, make = setup(dtype, head_dim=64, B=6, L=50, N=7, gamma=3)
    a = cached.run(*make(), prompts, lens, ud, uv, 3, 1.0)
    b = cached.run(*make(), prompts, lens, ud, uv, 3, 1.0, graph=True)
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_branches_of_one_context(dtype):
    """A prompt goes into one sequence, which is forked; the branches take different tokens, and each sees what a sequence of its
    own would: the same logits bit for bit.  Then the pages are compacted, and nothing changes."""
    w, _ = wl.attention_models(256, dtype, 3, 2, 4, 2, 64, device="cuda")
    B, L, n = 4, 37, 3
    g = torch.Generator(device="cuda").manual_seed(4)
    prompt = torch.randint(256, (1, L), dtype=torch.int32, device="cuda", generator=g).expand(B, L).contiguous()
    blocks = torch.randint(256, (B, n), dtype=torch.int32, device="cuda", generator=g)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")        # noqa: E731
    apart, forked = cached.Decoder(w, B, 64), cached.Decoder(w, B, 64)
    apart.cache.extend(L)
    apart.forward(prompt, apart.cache.lens)
    new = forked.cache.extend(L, i32([L, 0, 0, 0]))
    forked.forward(prompt, forked.cache.lens, new)
    assert forked.cache.fork(i32([0, 0, 0]), i32([1, 2, 3])).tolist() == [0, 0, 0]
    assert int((forked.cache.refs > 0).sum()) == cp.ceil_div(L, 16) and int(forked.cache.refs.max()) == B
    logits = []
    for m in (apart, forked):
        assert m.cache.extend(n).tolist() == [n] * B
        logits.append(m.forward(blocks, m.cache.lens))
    assert torch.equal(*logits)
    # two branches end, the pages of the others move to the front
    forked.cache.truncate(i32([2**31 - 1, 0, 2**31 - 1, 0]))
    forked.cache.compact()
    used = int((forked.cache.refs > 0).sum())
    assert used == cp.ceil_div(L, 16) + 1 + (cp.ceil_div(L + n, 16) - cp.ceil_div(L, 16)) * 2 and bool((forked.cache.refs[:used] > 0).all())
    tok = i32([[5], [5], [7], [5]])
    for m in (apart, forked):
        m.cache.extend(1, i32([1, 0, 1, 0]))
    one = i32([1, 0, 1, 0])
    a, b = apart.forward(tok, apart.cache.lens, one), forked.forward(tok, forked.cache.lens, one)
    assert torch.equal(a[[0, 2]], b[[0, 2]])


def test_a_cache_that_is_full_is_reported():
    tw, dw, prompts, lens, ud, uv, make = setup(N=4, gamma=3)
    small = [cached.Decoder(w, 5, 42, 16) for w in (tw, dw)]
    with pytest.raises(RuntimeError, match="room"):
        cached.run(*small, prompts, lens, ud, uv, 3)
