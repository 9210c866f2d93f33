"""Prompts, rotary positions and cut rows without a GPU: what the entry points refuse before they touch a device, frequencies, and the plain forms that the
GPU tests compare with, pinned on cases worked out by hand."""
import ctypes
import math
import struct

import pytest
import torch

import paper_2403_10444_b200 as bv
import prompt_plain as pp
from paper_2403_10444_b200 import build as bv_build

CACHE = struct.Struct("@5Q6q8i")


@pytest.fixture(scope="module")
def lib():
    bv_build.build()
    return bv.load_library()


@pytest.fixture(scope="module")
def at():
    buf = (ctypes.c_float * 64)()
    at.keep = buf
    return ctypes.addressof(buf) + -ctypes.addressof(buf) % 16


def rotary(lib, p, **bad):
    m = dict(k=p, v=p, table=p, lens=p, ks=(64, 32, 8), B=2, width=3, P=4, page=4, heads=2, D=8, dtype=0, freq=p, rot=8, side=0, mscale=1.0, q=p, out=p, kn=p, vn=p, new=None, off=None, n=2, q_heads=4,
             ok=None, st=(32, 16, 8), cache=True, rotary=True, qs=True)
    m.update(bad)
    cache = CACHE.pack(m["k"], m["v"], m["table"], m["lens"], 0, *m["ks"], *m["ks"], m["B"], m["width"], m["P"], m["page"], m["heads"], m["D"], m["dtype"], 0) if m["cache"] else None
    rot = struct.pack("@Qiifi", m["freq"], m["rot"], m["side"], m["mscale"], 0) if m["rotary"] else None
    st = struct.pack("@3q", *m["st"])
    qs = st if m["qs"] else None
    return lib.bv_cache_append_rotary(cache, rot, m["q"], qs, m["q_heads"], m["kn"], st, m["vn"], st, m["new"], m["off"], m["n"], m["out"], qs, m["ok"], st, None)


def prompt(lib, p, **bad):
    m = dict(q=p, k=p, v=p, off=p, B=2, tokens=3, q_heads=4, heads=2, D=8, dtype=0, scale=1.0, window=0, sinks=0, out=p, st=(32, 8), qs=True)
    m.update(bad)
    st = struct.pack("@2q", *m["st"])
    return lib.bv_prompt_attend(m["q"], st if m["qs"] else None, m["k"], st, m["v"], st, m["off"], m["B"], m["tokens"], m["q_heads"], m["heads"], m["D"], m["dtype"], ctypes.c_float(m["scale"]),
                                m["window"], m["sinks"], m["out"], st, None)


def sample(lib, x, **bad):
    m = dict(z=x, stride=8, u=x, rows=2, V=8, dtype=0, T=1.0, k=0, p=1.0, m=0.0, Ts=0, ks=0, ps=0, ms=0, tokens=x, lse=x, out=x, out_stride=8, cut=True)
    m.update(bad)
    cut = struct.pack("@4Qfiff", m["Ts"], m["ks"], m["ps"], m["ms"], m["T"], m["k"], m["p"], m["m"]) if m["cut"] else None
    return lib.bv_sample_filtered(m["z"], m["stride"], m["u"], m["rows"], m["V"], m["dtype"], cut, m["tokens"], m["lse"], m["out"], m["out_stride"], None)


def test_refusals_before_a_device_is_touched(lib, at):
    p = at
    for bad in (dict(k=0), dict(v=0), dict(table=0), dict(lens=2), dict(B=-1), dict(width=0), dict(P=0), dict(page=0), dict(heads=0), dict(D=0), dict(dtype=2), dict(ks=(64, -1, 8)), dict(cache=False),
                dict(rotary=False), dict(freq=0), dict(freq=p + 4), dict(rot=0), dict(rot=3), dict(rot=10), dict(mscale=math.nan), dict(mscale=math.inf), dict(q=None), dict(out=None), dict(q=p + 2),
                dict(qs=False), dict(q_heads=-1), dict(kn=None), dict(vn=p + 2), dict(st=(32, -16, 8)), dict(ok=p + 2), dict(n=0), dict(new=p + 2), dict(new=p, off=p), dict(off=p + 2)):
        assert rotary(lib, p, **bad) == -1, bad
    assert rotary(lib, p, q_heads=65533) == -2 and rotary(lib, p, D=4097) == -2
    assert rotary(lib, p, B=0) == 0 and rotary(lib, p, off=p, n=0) == 0
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(off=None), dict(out=None), dict(qs=False), dict(B=-1), dict(tokens=-1), dict(q_heads=3), dict(q_heads=0), dict(heads=0), dict(D=0),
                dict(dtype=2), dict(scale=math.nan), dict(scale=math.inf), dict(scale=3e38), dict(window=-1), dict(sinks=-1), dict(q=p + 2), dict(out=p + 2), dict(off=p + 2), dict(st=(-32, 8))):
        assert prompt(lib, p, **bad) == -1, bad
    assert prompt(lib, p, D=257) == -2 and prompt(lib, p, tokens=(1 << 30) + 1) == -2 and prompt(lib, p, B=(1 << 20) + 1) == -2 and prompt(lib, p, tokens=1 << 30) == -2
    assert prompt(lib, p, B=0) == 0 and prompt(lib, p, tokens=0) == 0
    for bad in (dict(z=None), dict(cut=False), dict(rows=-1), dict(V=0), dict(stride=-1), dict(out_stride=-1), dict(out_stride=7), dict(dtype=2), dict(u=None), dict(tokens=None),
                dict(u=None, tokens=None), dict(u=None, tokens=None, lse=None, out=None), dict(z=p + 2), dict(out=p + 2), dict(u=p + 2), dict(Ts=p + 2), dict(ks=p + 1), dict(T=0.0), dict(T=-1.0),
                dict(T=math.inf), dict(T=math.nan), dict(p=-0.5), dict(p=math.nan), dict(m=-0.1), dict(m=1.5), dict(m=math.nan)):
        assert sample(lib, p, **bad) == -1, bad
    assert sample(lib, p, V=(1 << 26) + 1, out=None) == -2 and sample(lib, p, rows=0) == 0
    # (a setting of its own for each row is not looked at here)
    assert sample(lib, p, rows=0, T=0.0, Ts=p) == 0


def test_frequencies():
    f = bv.rotary_frequencies(8, 10000.0, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(bv.rotary_frequencies(8, factor=4.0, device="cpu"), f / 4)
    # over 1000 positions the pairs turn 159, 16, 1.6 and 0.16 times: the first is as it was, the last a quarter, those between in between
    g = bv.rotary_frequencies(8, factor=4.0, original=1000, device="cpu")
    assert g[0] == f[0] and g[3] == f[3] / 4 and f[1] / 4 <= g[1] <= f[1] and f[2] / 4 <= g[2] <= f[2]
    for bad in (dict(rot=3), dict(rot=0), dict(rot=8, base=0.0), dict(rot=8, factor=0.0), dict(rot=8, factor=2.0, original=100, low=4.0, high=2.0)):
        with pytest.raises(ValueError):
            bv.rotary_frequencies(**bad, device="cpu")


def test_the_plain_rotation_by_hand():
    x = torch.tensor([[1.0, 2.0, 3.0, 4.0, 5.0]])
    quarter = torch.tensor([math.pi / 2, 0.0], dtype=torch.float64)
    y, _ = pp.rotate(x, torch.tensor(1), quarter, False, 2.0)
    assert torch.allclose(y, torch.tensor([[-6.0, 4.0, 2.0, 8.0, 5.0]], dtype=torch.float64))
    y, _ = pp.rotate(x, torch.tensor(1), quarter, True, 1.0)
    assert torch.allclose(y, torch.tensor([[-2.0, 1.0, 3.0, 4.0, 5.0]], dtype=torch.float64))


def test_the_plain_attention_by_loops():
    g = torch.Generator().manual_seed(1)
    q, k, v = torch.randn((9, 4, 8), generator=g), torch.randn((9, 2, 8), generator=g), torch.randn((9, 2, 8), generator=g)
    off = torch.tensor([1, 6, 6, 8])
    out, bound, written = pp.attend(q, k, v, off, window=3, sinks=1)
    assert written.tolist() == [False] + [True] * 7 + [False]
    for first, end in ((1, 6), (6, 8)):
        for i in range(first, end):
            seen = [j for j in range(first, i + 1) if i - j < 3 or j - first < 1]
            for h in range(4):
                w = torch.stack([q[i, h].double() @ k[j, h // 2].double() for j in seen]) * 8 ** -0.5
                w = (w - w.max()).exp()
                assert torch.allclose(out[i, h], sum(x * v[j, h // 2].double() for x, j in zip(w, seen)) / w.sum())
    assert bool((bound[1:8] > 0).all())


def test_the_plain_cut_by_hand():
    z = torch.log(torch.tensor([0.1, 0.4, 0.2, 0.2, 0.1]))
    keeps = lambda **c: pp.cut(z, **c)[0].tolist()      # noqa: E731
    assert keeps() == [True] * 5 and keeps(top_k=3) == [False, True, True, True, False] and keeps(top_k=2) == [False, True, True, False, False]
    assert keeps(top_p=0.3) == [False, True, False, False, False] and keeps(top_p=0.5) == [False, True, True, False, False] and keeps(top_p=0.0) == [False, True, False, False, False]
    assert keeps(min_p=0.4) == [False, True, True, True, False] and keeps(top_k=2, top_p=0.7) == [False, True, True, False, False]      # (0.4 of 0.6 is less than 0.7 of it)
    assert pp.cut(torch.tensor([1.0, math.nan])) is None and pp.cut(torch.tensor([-math.inf])) is None
    _, w = pp.cut(z, top_k=3)
    assert pp.drawn(w, 0.1) == (1, True) and pp.drawn(w, 0.0)[0] == 1 and pp.drawn(w, 0.6)[0] == 2 and pp.drawn(w, 0.8)[0] == 3 and pp.drawn(w, 0.999)[0] == 3
