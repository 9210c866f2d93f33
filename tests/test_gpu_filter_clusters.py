"""Rows that several CTAs share, cut to few tokens: every bit as sorting has it, again and again, with other calls' CTAs on the same multiprocessors."""
import pytest
import torch

import paper_2403_10444_b200 as bv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def plain(z, u, k):
    """(rows cut to the k largest, tokens, where the uniform is clear of a border) by sorting in 64 bits; k int64 [rows, 1]."""
    order = z.sort(dim=1, descending=True, stable=True).indices
    kept = torch.zeros_like(z, dtype=torch.bool).scatter_(1, order, torch.arange(z.shape[1], device=z.device)[None, :] < k)
    cut = torch.where(kept, z, torch.full_like(z, -float("inf")))
    w = torch.where(kept, (z.double() - z.double().amax(1, keepdim=True)).exp(), 0.0)
    c = w.cumsum(1)
    t = u.double()[:, None] * c[:, -1:]
    tokens = ((c > t) & kept).to(torch.int32).argmax(1).to(torch.int32)
    # (the borders of the cells are the sums at kept tokens; both sides' sums are off by some 10^-13)
    clear = torch.where(kept, (c - t).abs(), 1.0).amin(1) > 1e-11
    return cut, tokens, clear


def check(z, u, k, got):
    cut, tokens, clear = plain(z, u, k)
    assert torch.equal(got[0], cut)
    assert bool((got[1] == tokens)[clear].all()) and bool(cut.gather(1, got[1].long()[:, None]).isfinite().all())


# (rows, V, type, settings of each row's own): one row of eight CTAs, rows of two and of four, as many of them as the rules give several CTAs
SHAPES = [(1, 32000, BF16, False), (1, 32000, F32, False), (16, 32000, BF16, False), (100, 50257, BF16, False), (100, 128256, BF16, False), (100, 50257, F32, False),
          (140, 128256, BF16, True), (300, 50257, F32, True), (30, 33000, F32, True)]


@pytest.mark.parametrize("rows,V,dtype,each", SHAPES)
def test_few_tokens_of_rows_that_several_ctas_share(rows, V, dtype, each):
    gen = torch.Generator(device="cuda").manual_seed(rows + V)
    side = torch.cuda.Stream()
    for law, sizes in ((lambda x: x * 3, (1, 2, 17, 50, 128)), (lambda x: (x * 4).round() / 2, (3, 50))):
        z = law(torch.randn((rows, V), device="cuda", generator=gen)).to(dtype)
        u = torch.rand((rows,), device="cuda", generator=gen)
        for k in sizes:
            ks = torch.randint(1, k + 1, (rows,), device="cuda", generator=gen, dtype=torch.int32) if each else torch.full((rows,), k, dtype=torch.int32, device="cuda")
            outs = [torch.full_like(z, 5.0) for _ in range(4)]
            tokens = []
            torch.cuda.synchronize()
            for i, out in enumerate(outs):
                tokens.append(bv.bv_sample_filtered(z, u, top_k=ks if each else k, out_logits=out, stream=side if i % 2 else None)[0])
            torch.cuda.synchronize()
            check(z, u, ks.long()[:, None], (outs[0], tokens[0]))
            assert all(torch.equal(o, outs[0]) for o in outs) and all(torch.equal(t, tokens[0]) for t in tokens)


def test_two_hundred_calls_side_by_side():
    """The commonest call, one row of some tens of thousands on eight CTAs: four streams at once, new rows every time."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = (torch.randn((200, 32000), device="cuda", generator=gen) * 3).to(BF16)
    u = torch.rand((200,), device="cuda", generator=gen)
    out, streams = torch.full_like(z, 5.0), [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    tokens = [bv.bv_sample_filtered(z[i:i + 1], u[i:i + 1], top_k=50, out_logits=out[i:i + 1], stream=streams[i % 4])[0] for i in range(200)]
    torch.cuda.synchronize()
    check(z, u, torch.full((200, 1), 50, device="cuda"), (out, torch.cat(tokens)))
