"""Rows of logits cut by top-k, top-p and min-p, and tokens drawn from them, against sorting in 64 bits (prompt_plain.cut): exact but for uniforms and
borders within 10^-11."""
import math

import pytest
import torch

import paper_2403_10444_b200 as bv
import prompt_plain as pp

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def rows_of(rows, V, dtype, law, seed=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((rows, V), generator=g)
    if law == "zipf":
        z = z * 0.3 - 1.1 * torch.log(torch.arange(1, V + 1).float())[torch.rand((rows, V), generator=g).argsort(1)]
    elif law == "wide":
        z = z * 3
    elif law == "steps":                           # many equal values, zeros of both signs
        z = (z * 2).round() / 2
        z[z == 0] = torch.where(torch.rand((int((z == 0).sum()),), generator=g) < 0.5, 0.0, -0.0)
    elif law == "masked":
        z = torch.where(torch.rand((rows, V), generator=g) < 0.7, torch.tensor(-math.inf), z * 3)
        z[:, V // 2] = 1.0
    elif law == "low":
        z = torch.where(torch.rand((rows, V), generator=g) < 0.5, torch.tensor(torch.finfo(dtype).min), z)
        z[:, 0] = -1e4
    elif law == "equal":
        z = torch.full((rows, V), -2.5)
    return z.to(dtype).cuda()


def check(z, u, out=None, **cut):
    rows, V = z.shape
    keep = z.clone()
    filtered = torch.full_like(z, 5.0) if out is None else out
    tokens, lse = bv.bv_sample_filtered(z, u, out_logits=filtered, **cut)
    assert bv.bv_last_launch_count() == 1
    each = lambda name, i, d: (cut[name][i].item() if isinstance(cut.get(name), torch.Tensor) else cut.get(name, d))      # noqa: E731
    for r in range(rows):
        T = each("temperature", r, 1.0)
        known = pp.cut(keep[r], T, each("top_k", r, 0), each("top_p", r, 1.0), each("min_p", r, 0.0))
        if known is None:
            assert tokens[r].item() == -1 and math.isnan(lse[r].item())
            assert torch.equal(filtered[r].isnan(), keep[r].isnan()) and torch.equal(filtered[r].nan_to_num(0.5, 1.5), keep[r].nan_to_num(0.5, 1.5))
            continue
        kept, w = known
        want = torch.where(kept.cuda(), keep[r], torch.full_like(keep[r], -math.inf))
        assert torch.equal(filtered[r], want), (r, int(kept.sum()), int((filtered[r] > -math.inf).sum()))
        token, clear = pp.drawn(w, u[r].double().item())
        if clear:
            assert tokens[r].item() == token, r
        want = keep[r].double().max().item() / float(torch.tensor(T, dtype=F32)) + math.log(w.sum())
        assert abs(lse[r].item() - want) <= 2.0 ** -24 * abs(want) + 1e-12
    assert torch.equal(z.nan_to_num(0.5), keep.nan_to_num(0.5)) or out is z
    if out is None:
        assert torch.equal(bv.bv_filter_logits(z, **cut).nan_to_num(7.0, 8.0), filtered.nan_to_num(7.0, 8.0))
        again, _ = bv.bv_sample_filtered(z, u, want_lse=False, **cut)
        assert torch.equal(again, tokens)
    return tokens


def uniforms(rows, seed=1):
    return torch.rand((rows,), generator=torch.Generator().manual_seed(seed)).cuda()


CUTS = [dict(), dict(top_k=1), dict(top_k=7), dict(top_k=50, top_p=0.95, temperature=0.7), dict(top_p=0.9, temperature=0.8), dict(top_p=0.5), dict(min_p=0.05), dict(min_p=1.0),
        dict(top_k=300, top_p=0.99, min_p=0.01, temperature=1.3), dict(top_p=0.0), dict(top_p=1e-6), dict(top_p=0.9999999), dict(top_k=10**6, top_p=1.5), dict(temperature=0.05, top_p=0.9)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("law", ["zipf", "wide", "flat", "steps", "masked", "low", "equal"])
@pytest.mark.parametrize("V", [1, 2, 37, 1000, 5003])
def test_cuts(law, dtype, V):
    z = rows_of(4, V, dtype, law, seed=V)
    for i, cut in enumerate(CUTS):
        check(z, uniforms(4, i), **cut)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V", [(1, 32000), (1, 128256), (3, 50257), (160, 4097), (2, 256000), (1, 300001), (1, 700000)])
def test_sizes(rows, V, dtype):
    """Every number of CTAs and of vectors a thread, and rows that no CTA holds."""
    for i, (law, cut) in enumerate((("zipf", dict(top_k=50, top_p=0.9, temperature=0.8)), ("wide", dict(top_p=0.97)), ("flat", dict(top_k=2000, min_p=0.3)), ("steps", dict(top_p=0.6)))):
        check(rows_of(rows, V, dtype, law, seed=i), uniforms(rows, i), **cut)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_row_of_its_own_settings(dtype):
    z = rows_of(40, 3001, dtype, "zipf")
    some = ((1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (0.6, 20, 0.95, 0.0), (1.2, 200, 0.9, 0.02), (1.0, 1, 1.0, 0.0), (3.0, -5, 2.0, 1.0))
    t, k, p, m = zip(*(some[i % 8] for i in range(40)))
    f = lambda x: torch.tensor(x, dtype=F32, device="cuda")      # noqa: E731
    arrays = dict(temperature=f(t), top_k=torch.tensor(k, dtype=torch.int32, device="cuda"), top_p=f(p), min_p=f(m))
    check(z, uniforms(40), **arrays)
    for name in arrays:
        check(z, uniforms(40), **{name: arrays[name]})


def test_settings_out_of_range_in_a_row():
    z = rows_of(8, 500, BF16, "wide")
    f = lambda *x: torch.tensor(x, dtype=F32, device="cuda")      # noqa: E731
    t = f(1.0, 0.0, -1.0, math.inf, math.nan, 1.0, 1.0, 1.0)
    p = f(0.9, 0.9, 0.9, 0.9, 0.9, -0.1, math.nan, 0.9)
    m = f(0, 0, 0, 0, 0, 0, 0, 1.5)
    out = torch.zeros_like(z)
    tokens, lse = bv.bv_sample_filtered(z, uniforms(8), temperature=t, top_p=p, min_p=m, out_logits=out)
    assert tokens.tolist()[1:] == [-1] * 7 and tokens[0] >= 0 and bool(lse[1:].isnan().all()) and bool(out[1:].isnan().all()) and not bool(out[0].isnan().any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1000, 4097])
def test_rows_that_cannot_be_read(dtype, V):
    z = rows_of(6, V, dtype, "wide")
    z[1, 3], z[2, V - 1], z[3], z[4, 0], z[4, 1] = math.nan, math.inf, -math.inf, math.inf, math.nan
    for cut in (dict(), dict(top_k=5), dict(top_p=0.9, min_p=0.1)):
        check(z, uniforms(6), **cut)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_places_and_strides(dtype):
    for V, width, start in ((1000, 1003, 0), (1000, 1016, 8), (999, 1024, 1), (4096, 4104, 4)):
        x = rows_of(5, width, dtype, "zipf")
        z = x[:, start:start + V]
        out = torch.full((5, width + 16), 9.0, dtype=dtype, device="cuda")[:, 8:8 + V]
        check(z, uniforms(5), out=out, top_k=40, top_p=0.9)
    # one row for all, expanded; in place
    z = rows_of(1, 2000, dtype, "zipf").expand(6, -1)
    check(z, uniforms(6), top_p=0.8)
    z = rows_of(6, 2001, dtype, "zipf")
    check(z, uniforms(6), out=z, top_k=100, top_p=0.9)
    z = rows_of(1, 300001, dtype, "wide")
    check(z, uniforms(1), out=z, top_p=0.9)


def test_the_uniforms_ends():
    z = rows_of(3, 4096, BF16, "zipf")
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 0.5], device="cuda")
    for cut in (dict(), dict(top_k=3), dict(top_p=0.5), dict(min_p=0.2)):
        check(z, u, **cut)


def test_all_kept_is_the_drafting_step():
    """Without a cut: the tokens and normalisers of bv_sample_draft, but for uniforms near a border of its 32-bit weights."""
    z = rows_of(64, 32000, BF16, "zipf")
    u = uniforms(64)
    a, la = bv.bv_sample_filtered(z, u, temperature=0.8)
    b, lb = bv.bv_sample_draft(z, u, 0.8)
    assert (a != b).sum() <= 2 and (la - lb).abs().max() < 3e-6


def test_the_law_of_the_tokens():
    """A million draws from a cut row of twenty tokens: each share within five standard deviations."""
    z = torch.linspace(2, -2, 20)[torch.randperm(20, generator=torch.Generator().manual_seed(0))].cuda()
    n = 1 << 20
    tokens, _ = bv.bv_sample_filtered(z[None].expand(n, -1), torch.rand((n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)), temperature=0.9, top_k=12, top_p=0.9)
    _, w = pp.cut(z, 0.9, 12, 0.9)
    share = torch.bincount(tokens.cpu().long(), minlength=20).double() / n
    w = w / w.sum()
    assert bool(((share - w).abs() <= 5 * (w * (1 - w) / n).sqrt()).all())


def test_captured_and_on_another_stream():
    z = rows_of(20, 32000, BF16, "zipf")
    u = uniforms(20)
    want, lse = bv.bv_sample_filtered(z, u, top_p=0.9, top_k=100)
    side, out = torch.cuda.Stream(), torch.empty_like(z)
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got, _ = bv.bv_sample_filtered(z, u, top_p=0.9, top_k=100, out_logits=out)
    z2 = z.roll(1, 0).clone()
    z.copy_(z2)
    u.copy_(u.roll(1, 0).clone())
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want.roll(1, 0)) and torch.equal(out, bv.bv_filter_logits(z2, top_p=0.9, top_k=100))
    got, _ = bv.bv_sample_filtered(z, u, top_p=0.9, top_k=100, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want.roll(1, 0))


def test_refusals():
    z, u = rows_of(3, 100, F32, "wide"), uniforms(3)
    f = torch.ones(3, device="cuda")
    for bad in (dict(z=z.half()), dict(z=z.cpu()), dict(z=z[0]), dict(z=z.t()), dict(u=u[:2]), dict(u=u.double()), dict(u=u.cpu()), dict(temperature=f.double()), dict(temperature=f[:2]),
                dict(top_k=f), dict(top_p=f.cpu()), dict(min_p=f[None]), dict(out_logits=z.bfloat16()), dict(out_logits=z[:, :50]), dict(out_logits=z[:1].expand(3, -1))):
        a = dict(z=z, u=u)
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            bv.bv_sample_filtered(a.pop("z"), a.pop("u"), **a)
    for bad in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan), dict(top_p=-0.1), dict(top_p=math.nan), dict(min_p=-1.0), dict(min_p=1.1),
                dict(min_p=math.nan)):
        with pytest.raises(bv.BVError):
            bv.bv_sample_filtered(z, u, **bad)
        with pytest.raises(bv.BVError):
            bv.bv_filter_logits(z, **bad)
    tokens, lse = bv.bv_sample_filtered(z[:0], u[:0])
    assert tokens.shape == (0,) and lse.shape == (0,) and bv.bv_filter_logits(z[:0]).shape == (0, 100)
