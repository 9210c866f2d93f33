"""Attention of packed prompts against the definition in 64 bits, with bounds by arithmetic (prompt_plain.attend)."""
import math

import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv
import prompt_plain as pp

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(lens, Hq, Hkv, D, dtype=BF16, head=0, tail=0, seed=0, q_scale=1.5, layout="one"):
    g = torch.Generator().manual_seed(seed)
    T = head + sum(lens) + tail
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g)
    x[:, :Hq] *= q_scale
    q, k, v = x.to(dtype).cuda().split([Hq, Hkv, Hkv], dim=1)
    if layout == "heads":                          # heads first in memory
        q, k, v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    off = torch.tensor([head + sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    return q, k, v, off


def check(q, k, v, off, window=0, sinks=0, scale=None, fill=3.0, bits=None):
    out = torch.full(q.shape, fill, dtype=q.dtype, device="cuda")
    got = bv.bv_prompt_attend(q, k, v, off, scale=scale, window=window, sinks=sinks, out=out)
    assert got is out and bv.bv_stream_status() == 0
    want, bound, written = pp.attend(q, k, v, off, scale, window, sinks, bits or (8 if q.dtype == BF16 else 24))
    g = got.double()
    assert torch.equal(torch.isnan(g) & written[:, None, None], torch.isnan(want))
    fine = written[:, None, None] & ~torch.isnan(want)
    same = torch.isinf(want) & (g == want)
    off_by = torch.where(same, torch.zeros_like(g), (g - want).abs() - bound)
    worst = off_by[fine].max().item() if fine.any() else 0.0
    assert worst <= 0, "off by %.3g more than the bound" % worst
    assert bool((g[~written] == fill).all())
    return got


SHAPES = [                                       # lengths, Hq, Hkv, D
    ([1], 1, 1, 64), ([45], 8, 8, 64), ([1, 2, 3], 4, 2, 128), ([127, 128, 129], 4, 4, 128), ([255, 257, 1], 8, 2, 64), ([31, 33, 64, 65], 32, 8, 128),
    ([300, 5, 0, 70], 14, 2, 80), ([200], 7, 1, 96), ([150, 90], 40, 8, 72), ([513], 3, 3, 112), ([77, 400], 10, 2, 16), ([60], 128, 1, 64), ([130], 65, 1, 32), ([9, 260], 24, 2, 120),
    ([1] * 30 + [20] * 5, 4, 1, 128), ([700], 2, 1, 128), ([40, 200], 4, 2, 33), ([90], 4, 2, 200), ([70, 3], 2, 1, 256), ([50], 130, 1, 64), ([1100], 1, 1, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_is_the_definition(shape, dtype):
    check(*make(*shape, dtype=dtype, seed=len(shape[0])))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("head,tail,layout", [(0, 5, "one"), (3, 200, "heads"), (130, 0, "one")])
def test_rows_of_no_sequence_stay(dtype, head, tail, layout):
    check(*make([100, 40, 1], 8, 2, 64, dtype=dtype, head=head, tail=tail, layout=layout))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (64, 4), (127, 17), (128, 0), (200, 150), (2**31 - 1, 3), (300, 2**31 - 1), (33, 300)])
def test_windows_and_sinks(dtype, window, sinks):
    check(*make([700, 130, 1, 260], 6, 2, 64, dtype=dtype, seed=window % 97), window=window, sinks=sinks)
    check(*make([300], 8, 1, 128, dtype=dtype, seed=window % 89), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, 1e-6, 1.0, -0.3, 3.0])
def test_scales(dtype, scale):
    check(*make([140, 33], 4, 2, 64, dtype=dtype, q_scale=1.0), scale=scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [1e2, 1e5, 1e10, 1e15])
def test_scores_of_every_size(dtype, size):
    """Rows of which one key has everything, whatever the sizes: that key's value."""
    q, k, v, off = make([200, 70], 4, 2, 64, dtype=dtype, q_scale=1.0)
    q.mul_(size)
    out = bv.bv_prompt_attend(q, k, v, off)
    assert bool(torch.isfinite(out).all())
    want, _, _ = pp.attend(q, k, v, off, weight_bits=8)
    # scores are sums of 64 products with 2^-24 each: keys within that of the largest share a row in any way
    s = torch.einsum("thd,jhd->htj", q.double(), k.double().repeat_interleave(2, 1)) / 8
    for first, end in ((0, 200), (200, 270)):
        x = s[:, first:end, first:end].masked_fill(torch.ones(end - first, end - first, device="cuda").triu(1).bool(), -math.inf)
        two = x.topk(2, -1).values if end - first > 1 else None
        sure = (two[..., 0] - two[..., 1] > 128 * 2.0 ** -24 * two[..., 0].abs().clamp_min(1) * 64 + 40).t()
        sure[0] = True
        got, w = out[first:end].double(), want[first:end]
        assert torch.equal(got[sure], w[sure].to(dtype).double())
        if size >= 1e5:
            assert sure.float().mean() > 0.5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_references_that_grow_and_fall(dtype):
    """Scores that rise by much from tile to tile (every tile scales what was before), or fall."""
    q, k, v, off = make([900, 700], 4, 2, 64, dtype=dtype, q_scale=0.2)
    ramp = torch.cat([torch.linspace(0, 12, 900), torch.linspace(12, 0, 700)]).cuda()
    q[..., 0] = 4.0
    k[..., 0] = ramp[:, None].to(dtype) * 8
    check(q, k, v, off)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window", [0, 70])
def test_what_is_not_seen_does_not_count(dtype, value, window):
    """Keys and values that are not finite, in rows of no sequence, in later tokens, before the window."""
    lens = [150, 300, 20]
    q, k, v, off = make(lens, 8, 2, 64, dtype=dtype, head=4, tail=140)
    clean = bv.bv_prompt_attend(q, k, v, off, window=window)
    bad_k, bad_v = k.clone(), v.clone()
    for t in (bad_k, bad_v):
        t[:4] = value
        t[474:] = value
    assert torch.equal(bv.bv_prompt_attend(q, bad_k, bad_v, off, window=window), clean)
    # tokens in the middle of a sequence: those before them, those whose windows are past them and the other sequences do not see them
    at = 4 + 150 + 131
    bad_v[at, 1, 5], bad_v[at + 1, 0, 7] = value, value
    got = bv.bv_prompt_attend(q, bad_k, bad_v, off, window=window)
    want = clean.clone()
    upto = 454 if not window else None
    for token, head, d in ((at, 1, 5), (at + 1, 0, 7)):
        end = upto or token + window
        want[token:end, 4 * head:4 * head + 4, d] = value
    if not math.isnan(value):
        assert torch.equal(got, want)
    else:
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(9.0), want.nan_to_num(9.0))
    # a key that is not finite: rows that see it are what the formula gives (NaN, or without it), others as they were
    bad_k = k.clone()
    bad_k[at] = value
    got = bv.bv_prompt_attend(q, bad_k, v, off, window=window)
    hit = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    hit[at:upto or at + window] = True
    assert torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_weight(dtype):
    """Scores of -inf weigh nothing; where all are, 0 / 0."""
    q, k, v, off = make([130, 10], 2, 1, 64, dtype=dtype)
    q[..., 0], k[:, :, 0] = 1.0, 0.0
    k[:100, :, 0] = -math.inf
    check(q, k, v, off)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_odd_strides_and_places(dtype):
    lens, Hq, Hkv, D = [150, 37], 6, 2, 64
    g = torch.Generator().manual_seed(3)
    x = torch.randn((187, 23, D + 1), generator=g).to(dtype).cuda()
    off = torch.tensor([0, 150, 187], dtype=torch.int32, device="cuda")
    q, k, v = x[:, 0:12:2, 1:], x[:, 12:14, :D], x[:, 15:17, 1:]
    want = bv.bv_prompt_attend(*(t.contiguous() for t in (q, k, v)), off)
    check(q, k, v, off)
    assert (bv.bv_prompt_attend(q, k, v, off).double() - want.double()).abs().max() < 0.05
    # one head of keys for all, expanded; an output with gaps
    k1, v1 = k[:, :1].expand(-1, 2, -1), v[:, :1].expand(-1, 2, -1)
    check(q, k1, v1, off)
    out = torch.zeros((187, 9, 80), dtype=dtype, device="cuda")
    bv.bv_prompt_attend(q, k, v, off, out=out[:, 1:7, 3:67])
    assert torch.equal(out[:, 1:7, 3:67], bv.bv_prompt_attend(q, k, v, off)) and not out[:, 0].any() and not out[..., 67:].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off", [[0, 0, 0], [5, 5], [0, 50, 30, 90], [-1, 20, 60], [0, 1000], [90, 90, 90, 100], [0, 2**31 - 1], [-2**31, 2**31 - 1, 40, 90]])
def test_offsets_that_are_none(dtype, off):
    q, k, v, _ = make([100], 4, 2, 64, dtype=dtype)
    check(q, k, v, torch.tensor(off, dtype=torch.int32, device="cuda"))


def test_many_sequences():
    """More than a launch's table holds, of all lengths, empty ones among them."""
    lens = [(i * 7919) % 23 for i in range(2500)]
    check(*make(lens, 2, 1, 64))
    check(*make([1] * 1024 + [200], 2, 2, 128))


def test_long():
    """Each row's last keys and its first ones, over many tiles; one head so that 64 bits hold it."""
    check(*make([4500], 1, 1, 128, q_scale=2.0))
    check(*make([2300, 10, 900], 2, 1, 64, q_scale=2.0), window=1024, sinks=4)


def test_the_same_as_over_the_cache():
    """A whole prompt's attention over its pages, and the packed one: the same within the rounding of both."""
    lens = [70, 200, 33]
    q, k, v, off = make(lens, 8, 2, 128)
    c = cp.make(3, 200, 8, 2, 128, 16, lens)
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qp, kp, vp = (torch.zeros((3, 200, t.shape[1], 128), dtype=BF16, device="cuda") for t in (q, k, v))
    for b, (m, o) in enumerate(zip(lens, off.tolist())):
        qp[b, :m], kp[b, :m], vp[b, :m] = q[o:o + m], k[o:o + m], v[o:o + m]
    bv.bv_cache_append(kp, vp, c.k, c.v, c.table, c.lens, n_new=new)
    paged = bv.bv_cache_attend(qp, c.k, c.v, c.table, c.lens, n_new=new)
    want, bound, _ = pp.attend(q, k, v, off, weight_bits=8)
    got = torch.cat([paged[b, :m] for b, m in enumerate(lens)])
    assert bool(((got.double() - want).abs() <= 2 * bound).all())
    check(q, k, v, off)


def test_the_same_bits_again_captured_and_beside_another():
    q, k, v, off = make([300, 5, 900], 16, 4, 128)
    want = bv.bv_prompt_attend(q, k, v, off)
    for _ in range(3):
        assert torch.equal(bv.bv_prompt_attend(q, k, v, off), want)
    side, out = torch.cuda.Stream(), torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bv.bv_prompt_attend(q, k, v, off, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        bv.bv_prompt_attend(q, k, v, off, out=out)
    # other lengths in a replay; calls on both streams at once
    off2 = torch.tensor([0, 1, 700, 1205], dtype=torch.int32, device="cuda")
    want2 = bv.bv_prompt_attend(q, k, v, off2)
    off.copy_(off2)
    out.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        g.replay()
        other = bv.bv_prompt_attend(q, k, v, off2)
        third = bv.bv_prompt_attend(q, k, v, off2, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want2) and torch.equal(other, want2) and torch.equal(third, want2)


def test_no_graph_is_left():
    q, k, v, off = make([30], 4, 2, 64)
    for t in (q, k, v):
        t.requires_grad_(True)
    got = bv.bv_prompt_attend(q, k, v, off)
    assert got.grad_fn is None and not got.requires_grad and "orward only" in bv.bv_prompt_attend.__doc__


@pytest.mark.parametrize("shape", [([45], 8, 8, 64), ([700, 30, 1], 8, 2, 128)])
def test_a_wait_that_runs_out_ends_the_call(bv_options, shape):
    q, k, v, off = make(*shape)
    want = bv.bv_prompt_attend(q, k, v, off)
    assert bv.bv_stream_status() == 0
    bv_options("wait_limit", 3000)
    bv_options("never_signal", 1)
    bv.bv_prompt_attend(q, k, v, off)
    assert bv.bv_stream_status() == -4
    bv.bv_set_option("never_signal", 0)
    bv.bv_set_option("wait_limit", 0)
    for _ in range(3):
        assert torch.equal(bv.bv_prompt_attend(q, k, v, off), want)
    assert bv.bv_stream_status() == 0


def test_refusals():
    q, k, v, off = make([30], 4, 2, 64)
    for bad in (dict(q=q[:20]), dict(k=k[:, :1]), dict(v=v.float()), dict(q=q.half(), k=k.half(), v=v.half()), dict(off=off.long()), dict(off=off.cpu()), dict(off=off[:0]), dict(off=off[None]),
                dict(out=q[:20]), dict(out=q[:1].expand(30, -1, -1)), dict(q=q[None]), dict(q=q.transpose(1, 2))):
        a = dict(q=q, k=k, v=v, off=off, out=None)
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            bv.bv_prompt_attend(a["q"], a["k"], a["v"], a["off"], out=a["out"])
    for bad in (dict(window=-1), dict(sinks=-1), dict(scale=math.nan), dict(scale=math.inf)):
        with pytest.raises(bv.BVError):
            bv.bv_prompt_attend(q, k, v, off, **bad)
    with pytest.raises(bv.BVError):
        bv.bv_prompt_attend(q[:, :3], k, v, off)
    big = torch.zeros((2, 1, 300), dtype=BF16, device="cuda")
    with pytest.raises(bv.BVError) as e:
        bv.bv_prompt_attend(big, big, big, off)
    assert e.value.status == -2
    # nothing to do
    empty = torch.zeros((1,), dtype=torch.int32, device="cuda")
    assert not bv.bv_prompt_attend(q, k, v, empty).any()
    assert bv.bv_prompt_attend(q[:0], k[:0], v[:0], off).shape == (0, 4, 64)


@pytest.mark.parametrize("lens,Hq,Hkv,D", [([700, 1, 0, 333, 129], 39, 13, 128), ([1], 1, 1, 68), ([130] * 9 + [127, 5], 32, 32, 100), ([2500], 16, 16, 96)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 7)])
def test_32_bits_with_tiles_for_every_multiprocessor(lens, Hq, Hkv, D, window, sinks):
    """More than 64 columns and many tiles (and one that has few): whatever tile's size is taken, hidden values that are not finite stay hidden."""
    q, k, v, off = make(lens, Hq, Hkv, D, dtype=F32, head=2, tail=3, seed=D)
    for t in (k, v):
        t[:2], t[-3:] = math.nan, math.inf
    if window and lens[0] > 300:
        v[2 + 50] = math.nan                       # rows 50 to 149 of the first sequence are NaN, no other
    check(q, k, v, off, window=window, sinks=sinks)


@pytest.mark.parametrize("lens,Hq,Hkv,D", [([1500, 3, 0, 2100, 64, 65, 900] + [7] * 40, 32, 8, 128), ([1] * 700, 16, 16, 64)])
def test_more_units_than_multiprocessors(bv_options, lens, Hq, Hkv, D):
    """Whichever CTA does a unit: the definition, the same bits every time, beside itself on another stream, and after a call that gave up."""
    q, k, v, off = make(lens, Hq, Hkv, D, head=1, tail=2, seed=D)
    want = check(q, k, v, off)
    side, outs = torch.cuda.Stream(), [torch.full_like(want, 3.0) for _ in range(6)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        bv.bv_prompt_attend(q, k, v, off, out=out, stream=side if i % 2 else None)
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out in outs)
    bv_options("wait_limit", 3000)
    bv_options("never_signal", 1)
    bv.bv_prompt_attend(q, k, v, off)
    assert bv.bv_stream_status() == -4
    bv.bv_set_option("never_signal", 0)
    bv.bv_set_option("wait_limit", 0)
    check(q, k, v, off)
    assert bv.bv_stream_status() == 0
