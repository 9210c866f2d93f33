"""Rotary positions on the way into the cache against 64 bits, with bounds by arithmetic (prompt_plain.rotate)."""
import math

import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv
import prompt_plain as pp

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def close(got, want, bound, mask=None):
    off = (got.double() - want).abs() - bound
    worst = (off if mask is None else off[mask]).max().item() if off.numel() else 0.0
    assert worst <= 0, "off by %.3g more than the bound" % worst


def check(c, freq, n_new=None, interleaved=False, mscale=1.0, q_view=None):
    """Blocks [B, n] that go into a cache; everything that is not written stays as it was."""
    B, n, Hq, D = c.q.shape
    k0, v0 = c.k.clone(), c.v.clone()
    new = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device="cuda")
    out = bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq, n_new=new, interleaved=interleaved, mscale=mscale)
    assert bv.bv_last_launch_count() == 1
    ms = [n] * B if n_new is None else [min(max(m, 0), n) for m in n_new]
    lens = c.lens.cpu().tolist()
    at = torch.tensor([[L - m + t for t in range(n)] for L, m in zip(lens, ms)], device="cuda")
    brought = torch.tensor([[t < m for t in range(n)] for m in ms], device="cuda")
    for x, got in ((c.q, out),):
        want, bound = pp.rotate(x, at, freq, interleaved, mscale)
        close(got, want, bound, brought[:, :, None, None].expand_as(got))
        if n_new is not None:
            assert not got[~brought].any()
    want, bound = pp.rotate(c.k_new, at, freq, interleaved, mscale)
    kw, kb, vw = k0.double(), torch.zeros_like(k0, dtype=torch.float64), v0.clone()
    for b in range(B):
        for t in range(ms[b]):
            p = int(at[b, t])
            page = int(c.table[b, p // c.page]) if p >= 0 else -1
            if page >= 0:
                kw[page, :, p % c.page], kb[page, :, p % c.page] = want[b, t], bound[b, t]
                vw[page, :, p % c.page] = c.v_new[b, t]
    close(c.k, kw, kb)
    assert torch.equal(c.v, vw)
    return out


# (B, n, Hq, Hkv, D, page, lengths), rot
SHAPES = [((1, 1, 1, 1, 64, 16, [1]), 64), ((1, 1, 8, 8, 64, 16, [1000]), 64), ((3, 9, 64, 8, 128, 32, [9, 700, 1025]), 128), ((2, 5, 10, 2, 80, 24, [5, 501]), 80),
          ((2, 5, 10, 2, 80, 24, [7, 77]), 36), ((2, 3, 4, 1, 33, 5, [4, 77]), 32), ((2, 2, 4, 2, 256, 8, [30, 90]), 64), ((2, 3, 6, 3, 96, 192, [191, 400]), 2),
          ((1, 4, 3, 1, 7, 4, [9]), 6), ((200, 1, 16, 4, 128, 16, [1 + 7 * i for i in range(200)]), 128), ((3, 17, 2, 1, 512, 4, [17, 20, 40]), 512)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,rot", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_blocks(shape, rot, dtype, interleaved):
    c = cp.make(*shape, dtype=dtype, layout="tokens" if interleaved else "heads", seed=rot)
    check(c, bv.rotary_frequencies(rot), interleaved=interleaved, mscale=1.0 if rot > 64 else 1.25)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_each_sequence_brings_its_own_number(dtype, interleaved):
    c = cp.make(6, 5, 4, 2, 64, 16, [40, 3, 5, 100, 17, 2], dtype=dtype)
    check(c, bv.rotary_frequencies(64), n_new=[5, 0, -3, 9, 1, 4], interleaved=interleaved)      # (the last one is longer than its sequence)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """Positions whose angles 32 bits do not hold."""
    lens = [2**31 - 1024, 131072, 1000003, 2**24 + 1]
    c = cp.make(4, 3, 4, 2, 64, 16, [64] * 4, dtype=F32)
    c.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    freq = bv.rotary_frequencies(64, 1e6)
    out = torch.empty_like(c.q)
    # (pages of 2^15 tokens that are none: nothing is stored, and the queries turn all the same)
    small = torch.zeros((1, 2, 1 << 15, 64), device="cuda")
    c.table = torch.full((4, 1 << 16), -1, dtype=torch.int32, device="cuda")
    bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, small, small.clone(), c.table, c.lens, freq, out_q=out, interleaved=interleaved)
    at = torch.tensor([[L - 3 + t for t in range(3)] for L in lens], device="cuda")
    close(out, *pp.rotate(c.q, at, freq, interleaved, 1.0))
    assert not small.any()


def packed(lens, Hq, Hkv, D, dtype, page=16, tail=0, head=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    T = head + sum(lens) + tail
    qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=g).to(dtype).cuda()
    off = torch.tensor([head + sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    return qkv.split([Hq, Hkv, Hkv], dim=1) + (off,)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,before,Hq,Hkv,D,rot,interleaved", [
    ([1], [0], 1, 1, 64, 64, False), ([5, 0, 33, 1], [0, 3, 16, 99], 8, 2, 128, 128, False), ([5, 0, 33, 1], [0, 3, 16, 99], 8, 2, 128, 128, True),
    ([17] * 70, [i for i in range(70)], 4, 4, 80, 40, False), ([300, 7], [1, 1000], 5, 1, 36, 36, True), ([2500], [0], 2, 2, 64, 32, False), ([1] * 1100, [5] * 1100, 2, 1, 64, 64, False)])
@pytest.mark.parametrize("inplace", [False, True])
def test_packed(lens, before, Hq, Hkv, D, rot, interleaved, dtype, inplace):
    q, kn, vn, off = packed(lens, Hq, Hkv, D, dtype, tail=3, head=2, seed=rot)
    c = cp.make(len(lens), 1, Hq, Hkv, D, 16, [x + y for x, y in zip(lens, before)], dtype=dtype)
    freq = bv.rotary_frequencies(rot, 5e5)
    at = torch.full((q.shape[0],), 0, device="cuda")
    b_of = torch.full((q.shape[0],), -1, dtype=torch.long, device="cuda")
    for b, (m, L, o) in enumerate(zip(lens, before, off.tolist())):
        at[o:o + m] = torch.arange(L, L + m, device="cuda")
        b_of[o:o + m] = b
    some = b_of >= 0
    wq, bq = pp.rotate(q, at, freq, interleaved, 1.5)
    wk, bk = pp.rotate(kn, at, freq, interleaved, 1.5)
    k0, v0, q0, kn0 = c.k.clone(), c.v.clone(), q.clone(), kn.clone()
    out_q = q if inplace else torch.full((q.shape[0] + 1, Hq + 1, D), 7.0, dtype=dtype, device="cuda")[:-1, :-1]      # (at strides of its own)
    out_k = kn if inplace else torch.full_like(kn, 7.0)
    got = bv.bv_cache_append_rotary(q, kn, vn, c.k, c.v, c.table, c.lens, freq, offsets=off, interleaved=interleaved, mscale=1.5, out_q=out_q, out_k=out_k)
    assert got is out_q
    close(out_q[some], wq[some], bq[some])
    close(out_k[some], wk[some], bk[some])
    rest = (q0, kn0) if inplace else (torch.full_like(out_q, 7.0), torch.full_like(out_k, 7.0))
    assert torch.equal(out_q[~some], rest[0][~some]) and torch.equal(out_k[~some], rest[1][~some])
    page = c.table.long()[b_of[some], at[some] // 16]
    kw, kb, vw = k0.double(), torch.zeros_like(k0, dtype=torch.float64), v0.clone()
    kw[page, :, at[some] % 16], kb[page, :, at[some] % 16], vw[page, :, at[some] % 16] = wk[some], bk[some], vn[some]
    close(c.k, kw, kb)
    assert torch.equal(c.v, vw)


def test_what_turns_is_what_was_to_be_stored():
    """In the pages and beside them, in blocks and packed: the same bits."""
    c = cp.make(4, 6, 8, 2, 128, 16, [6, 100, 33, 64])
    freq = bv.rotary_frequencies(128, factor=4.0, original=64)
    k2, v2 = c.k.clone(), c.v.clone()
    out = bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq)
    off = torch.arange(0, 25, 6, dtype=torch.int32, device="cuda")
    ok = torch.empty_like(c.k_new)
    again = bv.bv_cache_append_rotary(c.q.view(24, 8, 128), c.k_new.view(24, 2, 128), c.v_new.view(24, 2, 128), k2, v2, c.table, c.lens, freq, offsets=off, out_k=ok.view(24, 2, 128))
    assert torch.equal(out.view(24, 8, 128), again) and torch.equal(c.k, k2) and torch.equal(c.v, v2)
    for b, L in enumerate(c.lens.tolist()):
        for t in range(6):
            p = L - 6 + t
            assert torch.equal(c.k[c.table[b, p // 16], :, p % 16], ok[b, t])


def test_a_whole_turn_and_none():
    """Frequency 0 leaves everything as it was; position 0 too."""
    c = cp.make(2, 1, 4, 2, 64, 16, [1, 50])
    out = bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, torch.zeros(32, dtype=torch.float64, device="cuda"))
    assert torch.equal(out, c.q)
    out = bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, bv.rotary_frequencies(64))
    assert torch.equal(out[0], c.q[0]) and not torch.equal(out[1], c.q[1])


@pytest.mark.parametrize("bad", ["length", "page"])
def test_what_is_none_is_passed_over(bad):
    c = cp.make(3, 2, 4, 2, 64, 16, [40, 30, 20])
    freq = bv.rotary_frequencies(64)
    k0, v0 = c.k.clone(), c.v.clone()
    if bad == "length":
        c.lens[1] = -7
    else:
        c.table[1, 1] = 1000
    bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq)
    held = [c.table[b, (L - 1) // 16].item() for b, L in ((0, 40), (2, 20))]
    changed = [p for p in range(c.k.shape[0]) if not torch.equal(c.k[p], k0[p])]
    assert set(changed) == set(held)
    assert [p for p in range(c.v.shape[0]) if not torch.equal(c.v[p], v0[p])] == changed


def test_offsets_in_no_order():
    """Rows of sequences whose offsets are none, or that would be longer than their sequence, are not stored; the others are."""
    c = cp.make(4, 2, 4, 2, 64, 16, [40, 30, 20, 10])
    freq = bv.rotary_frequencies(64)
    k0 = c.k.clone()
    # rows 0 to 3 are the first's, 4 and 5 the third's or nobody's; the last one would be too long
    off = torch.tensor([0, 4, -3, 6, 2**31 - 1], dtype=torch.int32, device="cuda")
    bv.bv_cache_append_rotary(c.q.view(8, 4, 64), c.k_new.view(8, 2, 64), c.v_new.view(8, 2, 64), c.k, c.v, c.table, c.lens, freq, offsets=off)
    changed = [p for p in range(c.k.shape[0]) if not torch.equal(c.k[p], k0[p])]
    assert set(changed) <= {c.table[0, 2].item(), c.table[1, 1].item(), c.table[2, 1].item()}


def test_a_captured_call_and_another_stream():
    c = cp.make(3, 4, 4, 2, 64, 16, [40, 30, 20])
    freq = bv.rotary_frequencies(64)
    want = bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq)
    kw = c.k.clone()
    side, out = torch.cuda.Stream(), torch.empty_like(c.q)
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq, out_q=out)
    c.k.zero_()
    c.lens.add_(1)
    c.lens.sub_(1)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    for b, L in enumerate(c.lens.tolist()):
        assert torch.equal(c.k[c.table[b, (L - 1) // 16], :, (L - 1) % 16], kw[c.table[b, (L - 1) // 16], :, (L - 1) % 16])
    got = bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_keys_only_and_refusals():
    c = cp.make(2, 3, 4, 2, 64, 16, [40, 30])
    freq = bv.rotary_frequencies(64)
    k2, v2 = c.k.clone(), c.v.clone()
    bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq)
    assert bv.bv_cache_append_rotary(None, c.k_new, c.v_new, k2, v2, c.table, c.lens, freq) is None
    assert torch.equal(c.k, k2) and torch.equal(c.v, v2)
    off = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    for bad in (dict(freq=freq.float()), dict(freq=freq[:0]), dict(freq=freq.cpu()), dict(offsets=off), dict(offsets=off, n_new=off[:2]), dict(n_new=off), dict(out_q=c.q[:, :2]),
                dict(out_k=c.k_new[:1]), dict(out_k=c.k_new[:1].expand(2, -1, -1, -1)), dict(k_new=c.k_new[:, :2]), dict(q=c.q.float())):
        a = dict(q=c.q, k_new=c.k_new, v_new=c.v_new, freq=freq)
        a.update(bad)
        f = a.pop("freq")
        with pytest.raises(ValueError):
            bv.bv_cache_append_rotary(a.pop("q"), a.pop("k_new"), a.pop("v_new"), c.k, c.v, c.table, c.lens, f, **a)
    with pytest.raises(bv.BVError):
        bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, bv.rotary_frequencies(66))
    with pytest.raises(bv.BVError):
        bv.bv_cache_append_rotary(c.q, c.k_new, c.v_new, c.k, c.v, c.table, c.lens, freq, mscale=math.nan)
