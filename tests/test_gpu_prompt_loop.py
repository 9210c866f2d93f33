"""The decoding loop with packed prompts, rotary positions and cut distributions: against a loop that keeps no cache and forms every row of logits anew in
64 bits, cut by sorting; both ways of marshalling."""
import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv
import prompt_plain as pp
from paper_2403_10444_b200 import binding, cached, specdec, workloads as wl

pytestmark = pytest.mark.gpu


def dense_logits(w, tokens, window, sinks, rotary):
    """Logits after every token of one sequence, in float64: [L, V]."""
    x = w["embed"][tokens.long()].double()
    L, H, K, D = x.shape[0], w["heads"], w["kv_heads"], w["head_dim"]
    j = torch.arange(L, device=x.device)
    see = j[None, :] <= j[:, None]
    if window:
        see &= (j[None, :] > j[:, None] - window) | (j[None, :] < sinks)
    for layer in w["layers"]:
        qkv = (x @ layer["qkv"].double()).view(L, H + 2 * K, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:].repeat_interleave(H // K, 1)
        if rotary is not None:
            q, k = (pp.rotate(t, j, rotary.freq, rotary.interleaved, rotary.mscale)[0] for t in (q, k))
        s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(H // K, 1)) * D ** -0.5
        p = torch.softmax(s.masked_fill(~see, float("-inf")), -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(L, H * D) @ layer["out"].double()
    return x @ w["unembed"].double()


def cut_rows(z, T, cut):
    """Rows [..., V] with what is not kept at -inf, by sorting."""
    if cut is None:
        return z
    flat = z.reshape(-1, z.shape[-1])
    return torch.stack([r.masked_fill(~pp.cut(r, T, *cut)[0].to(r.device), float("-inf")) for r in flat]).view_as(z)


def plain_loop(tw, dw, prompts, lens, ud, uv, gamma, T, algo, window, sinks, rotary, cut):
    ctx = [prompts[b, :lens[b]].tolist() for b in range(prompts.shape[0])]
    start = [len(c) for c in ctx]
    dev = prompts.device
    last = lambda w, toks, n: cut_rows(torch.stack([dense_logits(w, torch.tensor(t, device=dev), window, sinks, rotary)[-n:] for t in toks]).float(), T, cut)      # noqa: E731
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


def setup(dtype="f32", V=512, B=5, L=40, N=4, gamma=3, seed=0, heads=4, kv_heads=2, head_dim=32, page=16, window=0, sinks=0, noise=0.05, rotary=None):
    tw, dw = wl.attention_models(V, dtype, seed, 2, heads, kv_heads, head_dim, noise, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    prompts = torch.randint(V, (B, L), dtype=torch.int32, device="cuda", generator=g)
    lens = torch.randint(1, L + 1, (B,), dtype=torch.int32, device="cuda", generator=g)
    lens[0], lens[1] = 1, L
    ud, uv = wl.loop_uniforms(N, B, gamma, seed + 1, "cuda")
    make = lambda: [cached.Decoder(w, B, L + N * (gamma + 1), page, window, sinks, rotary) for w in (tw, dw)]       # noqa: E731
    return tw, dw, prompts, lens, ud, uv, make


CASES = [("block_lse", 0, 0, 16, None, False), ("block", 9, 2, 5, cached.Cut(top_p=0.9), True), ("token_lse", 0, 0, 16, cached.Cut(40, 0.95, 0.02), False), ("token", 0, 0, 16, cached.Cut(top_k=5), True)]


@pytest.mark.parametrize("algo,window,sinks,page,cut,interleaved", CASES)
@pytest.mark.parametrize("packed", [False, True])
def test_the_loop_is_that_without_a_cache(algo, window, sinks, page, cut, interleaved, packed):
    rotary = cached.Rotary(bv.rotary_frequencies(32 if not interleaved else 16), interleaved, 1.0 if not interleaved else 1.1)
    tw, dw, prompts, lens, ud, uv, make = setup(window=window, sinks=sinks, page=page, rotary=rotary)
    res = cached.run(*make(), prompts, lens, ud, uv, 3, 0.9, algo, packed=packed, cut=cut)
    want = plain_loop(tw, dw, prompts, lens, ud, uv, 3, 0.9, algo, window, sinks, rotary, cut)
    for b, toks in enumerate(want):
        assert res["tokens"][b, :len(toks)].tolist() == toks and int(res["lengths"][b]) == len(toks)
        assert (res["tokens"][b, len(toks):] == -1).all()


@pytest.mark.parametrize("algo", specdec.ALGOS)
def test_cut_to_one_token_it_is_greedy(algo):
    """With top_k = 1 both models are certain, so the loop generates the target's likeliest tokens, whatever the uniforms are."""
    tw, dw, prompts, lens, ud, uv, make = setup()
    res = cached.run(*make(), prompts, lens, ud, uv, 3, 0.9, algo, cut=cached.Cut(top_k=1))
    for b in range(5):
        toks = prompts[b, :lens[b]].tolist()
        for _ in range(int(res["lengths"][b])):
            toks.append(int(dense_logits(tw, torch.tensor(toks, device="cuda"), 0, 0, None)[-1].argmax()))
        assert res["tokens"][b, :int(res["lengths"][b])].tolist() == toks[int(lens[b]):]


@pytest.mark.parametrize("dtype,head_dim,rotate", [("bf16", 64, True), ("bf16", 128, False), ("f32", 64, True)])
def test_packed_prompts_leave_the_same_cache(dtype, head_dim, rotate):
    """The first layer's keys and values bit for bit (the same products of the same rows are not asked of the library of products: so within one rounding), the
    others and the next logits within the roundings of the attention between: eps of the type, 2 layers, sums of a few terms of about one."""
    rotary = cached.Rotary(bv.rotary_frequencies(head_dim, factor=4.0, original=32)) if rotate else None
    tw, _, prompts, lens, _, _, make = setup(dtype, head_dim=head_dim, B=7, L=300, heads=8, rotary=rotary)
    a, b = make()[0], make()[0]
    for m, packed in ((a, False), (b, True)):
        assert torch.equal(m.cache.extend(300, lens), lens)
        if packed:
            off = torch.zeros((8,), dtype=torch.int32, device="cuda")
            off[1:] = lens.cumsum(0)
            held = torch.arange(300, device="cuda")[None, :] < lens[:, None]
            x = m.prefill(prompts[held], off)
            assert x.shape == (int(lens.sum()), 8 * head_dim)
        else:
            m.forward(prompts, m.cache.lens, lens)
    assert torch.equal(a.cache.table, b.cache.table)
    eps = torch.finfo(a.cache.k[0].dtype).eps
    for x, y in zip(a.cache.k + a.cache.v, b.cache.k + b.cache.v):
        assert (x - y).abs().max() <= 16 * eps * max(1.0, x.abs().max().item())
    i32 = dict(dtype=torch.int32, device="cuda")
    out = []
    for m in (a, b):
        m.cache.extend(1)
        out.append(m.forward(torch.full((7, 1), 3, **i32), m.cache.lens)[:, 0].float())
    assert (out[0] - out[1]).abs().max() <= 32 * eps * out[0].abs().max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replays_of_a_captured_iteration_give_the_same_tokens(dtype):
    rotary = cached.Rotary(bv.rotary_frequencies(64))
    tw, dw, prompts, lens, ud, uv, make = setup(dtype, head_dim=64, B=6, L=50, N=6, gamma=3, rotary=rotary)
    args = dict(packed=True, cut=cached.Cut(100, 0.9, 0.01))
    a = cached.run(*make(), prompts, lens, ud, uv, 3, 1.0, **args)
    b = cached.run(*make(), prompts, lens, ud, uv, 3, 1.0, graph=True, **args)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_prompts_of_one_token_each():
    tw, dw, prompts, lens, ud, uv, make = setup(L=3)
    lens.fill_(1)
    a = cached.run(*make(), prompts, lens, ud, uv, 3, 1.0)
    b = cached.run(*make(), prompts, lens, ud, uv, 3, 1.0, packed=True)
    assert torch.equal(a["tokens"], b["tokens"])


def test_both_ways_of_marshalling(monkeypatch):
    """The calls through the module in C++ and those checked in Python: the same results, in tensors of the same kind."""
    c = cp.make(3, 4, 8, 2, 64, 16, [40, 30, 20])
    freq = bv.rotary_frequencies(64)
    new = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 4, 4, 12], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(0)
    z, u = torch.randn((6, 999), generator=g).cuda(), torch.rand((6,), generator=g).cuda()
    flat = lambda t: t.reshape(12, t.shape[2], 64)      # noqa: E731
    some = torch.full((6,), 0.8, device="cuda")

    def calls():
        k, v = c.k.clone(), c.v.clone()
        r = [bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, k, v, c.table, c.lens, freq), bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, k, v, c.table, c.lens, freq, n_new=new, interleaved=True, mscale=2)]
        ok = torch.zeros_like(flat(c.k_new))
        r += [bv.bv_cache_append_rotary(flat(c.q), flat(c.k_new), flat(c.v_new), k, v, c.table, c.lens, freq, offsets=off, out_k=ok), ok, k, v]
        r += [bv.bv_prompt_attend(flat(c.q), flat(c.k_new), flat(c.v_new), off), bv.bv_prompt_attend(flat(c.q), flat(c.k_new), flat(c.v_new), off, scale=0.3, window=3, sinks=1)]
        r += list(bv.bv_sample_filtered(z, u, 0.9, 50, 0.9, 0.01)) + [bv.bv_sample_filtered(z, u, some, want_lse=False)[0], bv.bv_filter_logits(z, 1, 7), bv.bv_filter_logits(z, top_p=some)]
        return r

    fast = calls()
    assert binding._fast is not None
    monkeypatch.setattr(binding, "_fast", None)
    for x, y in zip(fast, calls()):
        assert torch.equal(x, y) and x.dtype == y.dtype and x.stride() == y.stride()
