"""The two ways in which a call of the cache is marshalled (the module _fast, and binding.py where that does not take it): the same
results, and the same refusals."""
import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv
from paper_2403_10444_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["fast", "interpreted"])
def way(request, monkeypatch):
    assert binding._fast is not None, "the module _fast is not built"
    if request.param == "interpreted":
        monkeypatch.setattr(binding, "_fast", None)
    return request.param


def everything(dtype):
    """All of the calls once, on one cache; what they return and leave."""
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                  # noqa: E731
    c = cp.make(4, 3, 8, 2, 64, 16, [33, 16, 70, 5], dtype=dtype, width=8, spare=20, seed=2)
    got = [bv.bv_pages_fork(c.table, c.lens, c.refs, 16, i32([0]), i32([3]))]
    got += bv.bv_pages_extend(c.table, c.lens, c.refs, 16, 3)
    bv.bv_pages_copy(c.k, c.v, got[-1])
    bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, c.table, c.lens)
    got.append(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens))
    got.append(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, n_new=i32([1, 0, 3, 2]), scale=0.3, window=20, sinks=2))
    got.append(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, out=torch.zeros_like(c.q)))
    got.append(bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, out=torch.zeros((3, 4, 8, 64), dtype=dtype, device="cuda").transpose(0, 1)).contiguous())
    bv.bv_pages_truncate(c.table, c.lens, c.refs, 16, i32([1, 3, 0, 2]), 3)
    bv.bv_pages_truncate(c.table, c.lens, c.refs, 16, i32([0, 99, 99, 99]))
    moves = bv.bv_pages_compact(c.table, c.lens, c.refs, 16)
    bv.bv_pages_copy(c.k, c.v, *moves)
    got += [*moves, *bv.bv_pages_extend(c.table, c.lens, c.refs, 16, 5, i32([5, 0, 2, 1]))]
    torch.cuda.synchronize()
    return got + [c.k, c.v, c.table, c.lens, c.refs]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_same_results(dtype, monkeypatch):
    fast = everything(dtype)
    monkeypatch.setattr(binding, "_fast", None)
    slow = everything(dtype)
    assert len(fast) == len(slow)
    for a, b in zip(fast, slow):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_the_same_refusals(way):
    c = cp.make(2, 3, 4, 2, 64, 16, [33, 16])
    args = lambda **x: {**dict(q=c.q, k=c.k, v=c.v, table=c.table, lens=c.lens), **x}   # noqa: E731
    for bad in (dict(q=c.q.float()), dict(q=c.q[:1]), dict(q=c.q[..., :32]), dict(table=c.table.long()), dict(lens=c.lens[:1]), dict(v=c.v[1:]), dict(k=c.k.transpose(2, 3)),
                dict(q=c.q.cpu()), dict(table=c.table.cpu(), lens=c.lens.cpu()), dict(n_new=c.lens[:1]), dict(out=c.q[:, :2]), dict(out=c.q[:, :1].expand_as(c.q))):
        with pytest.raises((ValueError, TypeError)):
            bv.bv_cache_attend(**args(**bad))
    for bad in (dict(scale=float("inf")), dict(window=-1), dict(sinks=-2), dict(q=c.q[:, :, :3])):
        with pytest.raises(bv.BVError) as err:
            bv.bv_cache_attend(**args(**bad))
        assert err.value.status == -1
    with pytest.raises(TypeError):
        bv.bv_cache_attend(**args(k=c.k.half(), v=c.v.half(), q=c.q.half()))
    with pytest.raises(bv.BVError):
        bv.bv_pages_extend(c.table, c.lens, c.refs, 16, 0)
    with pytest.raises(bv.BVError):
        bv.bv_pages_truncate(c.table, c.lens, c.refs, 16, c.lens, -1)
    with pytest.raises(ValueError):
        bv.bv_pages_truncate(c.table, c.lens, c.refs, 16, c.lens[:1])
    with pytest.raises(ValueError):
        bv.bv_pages_fork(c.table, c.lens, c.refs, 16, c.lens, c.lens[:1])
    with pytest.raises(ValueError):
        bv.bv_pages_copy(c.k, c.v, c.table)
    with pytest.raises(ValueError):
        bv.bv_cache_append(c.k_new, c.v_new[:, :2], c.k, c.v, c.table, c.lens)
    with pytest.raises(ValueError):
        bv.bv_cache_append(c.k_new, c.v_new, c.k[:1].expand_as(c.k), c.v, c.table, c.lens)
    assert bv.bv_pages_fork(c.table, c.lens, c.refs, 16, c.lens[:0], c.lens[:0]).shape == (0,)
    bv.bv_pages_copy(c.k, c.v, torch.zeros((0, 2), dtype=torch.int32, device="cuda"))


def test_another_stream(way):
    c = cp.make(2, 3, 4, 2, 64, 16, [33, 160])
    want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, stream=s)
    with torch.cuda.stream(s):
        again = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)


def test_what_is_made_for_a_call_belongs_to_its_stream(way):
    """The current stream is busy: neither the zeros of rows that a sequence does not bring, nor what lies in the memory before, may come after the result."""
    c = cp.make(2, 3, 4, 2, 64, 16, [33, 160], spare=20, width=16)
    new = torch.tensor([2, 3], dtype=torch.int32, device="cuda")
    want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, n_new=new)
    table, lens, refs = (x.clone() for x in (c.table, c.lens, c.refs))
    want_new, want_copies = bv.bv_pages_extend(table, lens, refs, 16, 3)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)                                                       # some 20 ms
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, n_new=new, stream=s)
    got_new, got_copies = bv.bv_pages_extend(c.table, c.lens, c.refs, 16, 3, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_new, want_new) and torch.equal(got_copies, want_copies)


def test_an_empty_batch(way):
    c = cp.make(2, 3, 4, 2, 64, 16, [33, 160])
    table, lens, k = c.table[:0], c.lens[:0], c.k.clone()
    assert bv.bv_cache_attend(c.q[:0], c.k, c.v, table, lens).shape == (0, 3, 4, 64)
    assert bv.bv_cache_attend(c.q[:0], c.k, c.v, table, lens, n_new=lens).shape == (0, 3, 4, 64)
    bv.bv_cache_append(c.k_new[:0], c.v_new[:0], c.k, c.v, table, lens)
    new, copies = bv.bv_pages_extend(table, lens, c.refs, 16, 3)
    assert new.shape == (0,) and copies.shape == (0, 2)
    bv.bv_pages_truncate(table, lens, c.refs, 16, lens)
    bv.bv_pages_copy(c.k, c.v, copies)
    torch.cuda.synchronize()
    assert torch.equal(c.k, k) and bv.bv_stream_status() == 0
