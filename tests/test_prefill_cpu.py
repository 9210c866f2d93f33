"""Where packed tokens of decoders without rotary positions go, and offsets that are refused before anything is indexed by them."""
import pytest
import torch

from paper_2403_10444_b200 import cached, workloads as wl


def decoder(B=3, capacity=20, page=4):
    tw, _ = wl.attention_models(16, "f32", 1, layers=1, heads=2, kv_heads=1, head_dim=4)
    return cached.Decoder(tw, B, capacity, page)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_places():
    m = decoder()
    m.cache.table[0, :2], m.cache.table[1, :1], m.cache.table[2, :3] = i32(7, 3), i32(5), i32(0, 9, 1)
    m.cache.lens.copy_(i32(6, 0, 9))
    # two rows of nobody, six of the first, three that the second has no room for, one of the third (its ninth), one of nobody
    table, lens = m._places(13, i32(2, 8, 11, 12))
    assert table.shape == (13, 1) and table.is_contiguous() and table.dtype == lens.dtype == torch.int32
    got = [(p, n) if n else None for (p,), n in zip(table.tolist(), lens.tolist())]
    assert got == [None] * 2 + [(7, 1), (7, 2), (7, 3), (7, 4), (3, 1), (3, 2)] + [None] * 3 + [(1, 1), None]
    # a length that is none, offsets in no order: nothing but places in range
    m.cache.lens.copy_(i32(21, -5, 2**31 - 1))
    assert not m._places(13, i32(2, 8, 11, 12))[1].any()
    m.cache.lens.copy_(i32(6, 6, 6))
    for offsets in (i32(0, 2**31 - 1, -2**31, 5), i32(9, 3, 1, 0), i32(-4, -2, 30, 40)):
        table, lens = m._places(13, offsets)
        assert bool(((lens >= 0) & (lens <= 4)).all())


def test_refusals():
    m = decoder()
    tokens = torch.zeros((5,), dtype=torch.int32)
    for offsets in (i32(0, 2, 5), i32(0, 2, 3, 4, 5), i32(0, 2, 3, 5).long(), i32(0, 2, 3, 5)[None]):
        with pytest.raises(ValueError):
            m.prefill(tokens, offsets)
    with pytest.raises(ValueError):
        m.prefill(tokens[None], i32(0, 2, 3, 5))
