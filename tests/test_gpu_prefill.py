"""Packed prompts of decoders without rotary positions: keys and values reach their pages as they are, whatever they hold and however wide a head is."""
import math

import pytest
import torch

import paper_2403_10444_b200 as bv
from paper_2403_10444_b200 import cached, workloads as wl

pytestmark = pytest.mark.gpu


def both(weights, tokens, lens, capacity, page=16):
    """The model after its prompts (tokens [B, L], the first lens[b] of a row) went through padded, and packed with some rows of no sequence around."""
    out = []
    B = tokens.shape[0]
    for packed in (False, True):
        m = cached.Decoder(weights, B, capacity, page)
        assert torch.equal(m.cache.extend(tokens.shape[1], lens), lens)
        if packed:
            offsets = torch.zeros((B + 1,), dtype=torch.int32, device="cuda")
            offsets[1:] = lens.cumsum(0)
            held = torch.arange(tokens.shape[1], device="cuda")[None, :] < lens[:, None]
            none = torch.full((3,), 2, dtype=torch.int32, device="cuda")
            m.prefill(torch.cat([none, tokens[held], none]), offsets + 3)
        else:
            m.forward(tokens, m.cache.lens, lens)
        out.append(m.cache)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_key_goes_into_its_page_alone(dtype):
    tw, _ = wl.attention_models(64, dtype, 1, layers=1, heads=4, kv_heads=2, device="cuda")
    # token 7 has 2^100 in a place where all others have 0, and element 1 of the first key takes it 2^100 times
    embed, qkv = tw["embed"], tw["layers"][0]["qkv"]
    embed[:, 5], embed[7], qkv[5] = 0.0, 0.0, 0.0
    embed[7, 5] = 2.0 ** 100
    qkv[5, 4 * 64 + 1] = 2.0 ** 100
    tokens = torch.randint(8, 64, (4, 50), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    tokens[:, 9] = 7
    lens = torch.tensor([50, 1, 10, 33], dtype=torch.int32, device="cuda")
    a, b = both(tw, tokens, lens, 50)
    assert torch.equal(a.table, b.table) and int((a.k[0] == math.inf).sum()) == 3
    for x, y in ((a.k[0], b.k[0]), (a.v[0], b.v[0])):
        assert torch.equal(x.isinf(), y.isinf()) and not bool(x.isnan().any()) and not bool(y.isnan().any())
        # (sums of 256 products of about one, in whatever order, rounded once)
        fine = ~x.isinf()
        assert (x - y)[fine].abs().max() <= 256 * 2.0 ** -23 * 16 + torch.finfo(x.dtype).eps * x[fine].abs().max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_dim,page", [(1, 16), (3, 5), (64, 1)])
def test_heads_of_any_width(dtype, head_dim, page):
    tw, _ = wl.attention_models(64, dtype, 1, layers=1, heads=4, kv_heads=2, head_dim=head_dim, device="cuda")
    tokens = torch.randint(64, (5, 40), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    lens = torch.tensor([40, 7, 0, 1, 39], dtype=torch.int32, device="cuda")
    a, b = both(tw, tokens, lens, 40, page)
    assert torch.equal(a.table, b.table)
    for x, y in zip(a.k + a.v, b.k + b.v):
        assert bool(x.any()) and (x - y).abs().max() <= 256 * 2.0 ** -23 * 16 + torch.finfo(x.dtype).eps * x.abs().max()


def test_prompts_that_found_no_room_are_not_stored():
    """A sequence without pages: its tokens go nowhere, the others' where they belong."""
    tw, _ = wl.attention_models(64, "f32", 1, layers=1, heads=4, kv_heads=2, device="cuda")
    m = cached.Decoder(tw, 3, 32)
    lens = torch.tensor([20, 32, 5], dtype=torch.int32, device="cuda")
    m.cache.extend(32, lens)
    m.cache.table[1], m.cache.lens[1] = -1, 0
    tokens = torch.randint(64, (57,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    offsets = torch.tensor([0, 20, 52, 57], dtype=torch.int32, device="cuda")
    m.prefill(tokens, offsets)
    stored = {int(p) for row in m.cache.table.tolist() for p in row if p >= 0}
    for x in m.cache.k + m.cache.v:
        used = x.abs().amax((1, 2, 3)) > 0
        assert {int(p) for p in used.nonzero()} == stored
