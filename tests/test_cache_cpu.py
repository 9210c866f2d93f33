"""The paged cache's entry points without a GPU: what they refuse before they touch a device, and the plain bookkeeping that the GPU
tests compare with, pinned on cases worked out by hand."""
import ctypes
import os
import struct
import subprocess

import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv
from paper_2403_10444_b200 import build as bv_build

CACHE = struct.Struct("@5Q6q8i")


@pytest.fixture(scope="module")
def lib():
    bv_build.build()
    return bv.load_library()


class Args:
    """A cache of two sequences that every call takes, to be spoilt one member at a time."""

    def __init__(self, **bad):
        self.buf = (ctypes.c_float * 64)()
        p = ctypes.addressof(self.buf) + -ctypes.addressof(self.buf) % 16
        m = dict(k=p, v=p, table=p, lens=p, refs=p, ks=(64, 32, 8), vs=(64, 32, 8), B=2, width=3, P=4, page=4, heads=2, D=8, dtype=0)
        self.bad = {x: y for x, y in bad.items() if x not in m}
        m.update({x: y for x, y in bad.items() if x in m})
        self.cache = CACHE.pack(m["k"], m["v"], m["table"], m["lens"], m["refs"], *m["ks"], *m["vs"], m["B"], m["width"], m["P"], m["page"], m["heads"], m["D"], m["dtype"], 0)
        self.p = p
        self.st = struct.pack("@3q", 32, 16, 8)


def attend(lib, **bad):
    a = Args(**bad)
    v = dict(q=a.p, qs=a.st, new=None, n=2, q_heads=4, scale=1.0, window=0, sinks=0, out=a.p, os=a.st)
    v.update(a.bad)
    return lib.bv_cache_attend(v.get("cache", a.cache), v["q"], v["qs"], v["new"], v["n"], v["q_heads"], ctypes.c_float(v["scale"]), v["window"], v["sinks"], v["out"], v["os"], None)


def append(lib, **bad):
    a = Args(**bad)
    v = dict(kn=a.p, kns=a.st, vn=a.p, vns=a.st, new=None, n=2)
    v.update(a.bad)
    return lib.bv_cache_append(v.get("cache", a.cache), v["kn"], v["kns"], v["vn"], v["vns"], v["new"], v["n"], None)


def extend(lib, **bad):
    a = Args(**bad)
    v = dict(new=None, n=2, out=a.p, copies=a.p)
    v.update(a.bad)
    return lib.bv_pages_extend(v.get("cache", a.cache), v["new"], v["n"], v["out"], v["copies"], None)


def truncate(lib, **bad):
    a = Args(**bad)
    v = dict(keep=a.p, new=None, n=0)
    v.update(a.bad)
    return lib.bv_pages_truncate(v.get("cache", a.cache), v["keep"], v["new"], v["n"], None)


def fork(lib, **bad):
    a = Args(**bad)
    v = dict(src=a.p, dst=a.p, forks=1, ok=a.p)
    v.update(a.bad)
    return lib.bv_pages_fork(v.get("cache", a.cache), v["src"], v["dst"], v["forks"], v["ok"], None)


def compact(lib, **bad):
    a = Args(**bad)
    v = dict(moves=a.p, count=a.p)
    v.update(a.bad)
    return lib.bv_pages_compact(v.get("cache", a.cache), v["moves"], v["count"], None)


def copy(lib, **bad):
    a = Args(**bad)
    v = dict(pairs=a.p, n=1, count=None)
    v.update(a.bad)
    return lib.bv_pages_copy(v.get("cache", a.cache), v["pairs"], v["n"], v["count"], None)


POOLS = [dict(k=0), dict(v=0), dict(k=2), dict(ks=(64, -1, 8)), dict(vs=(-64, 32, 8)), dict(heads=0), dict(D=0), dict(dtype=2), dict(P=0), dict(page=0), dict(cache=None)]
ROWS = [dict(table=0), dict(lens=0), dict(table=2), dict(lens=6), dict(B=-1), dict(width=0)]
COUNTS = [dict(refs=0), dict(refs=2), dict(P=0), dict(page=0), dict(cache=None)]


def test_refusals_before_a_device_is_touched(lib):
    odd = Args().p + 2
    neg = struct.pack("@3q", 32, -16, 8)
    for fn, bads in (
            (attend, POOLS + ROWS + [dict(q=None), dict(out=None), dict(qs=None), dict(os=None), dict(n=0), dict(heads=3), dict(q_heads=3), dict(q_heads=0), dict(window=-1), dict(sinks=-1),
                                     dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(scale=-3e38), dict(q=odd), dict(out=odd), dict(new=odd), dict(qs=neg), dict(os=neg)]),
            (append, POOLS + ROWS + [dict(kn=None), dict(vn=None), dict(kns=None), dict(vns=None), dict(n=0), dict(kn=odd), dict(new=odd), dict(kns=neg)]),
            (extend, ROWS + COUNTS + [dict(n=0), dict(out=None), dict(copies=None), dict(out=odd), dict(new=odd)]),
            (truncate, ROWS + COUNTS + [dict(keep=None), dict(keep=odd), dict(n=-1), dict(new=odd)]),
            (fork, ROWS + COUNTS + [dict(src=None), dict(dst=None), dict(ok=None), dict(forks=-1), dict(src=odd)]),
            (compact, ROWS + COUNTS + [dict(moves=None), dict(count=None), dict(moves=odd)]),
            (copy, POOLS + [dict(pairs=None), dict(n=-1), dict(pairs=odd), dict(count=odd)])):
        for bad in bads:
            assert fn(lib, **bad) == -1, (fn.__name__, bad)
    # larger than what is built
    assert attend(lib, D=257) == -2 and attend(lib, n=2**30, q_heads=4) == -2
    assert extend(lib, B=8193) == -2 and extend(lib, P=1 << 22) == -2 and truncate(lib, B=1 << 16) == -2
    assert copy(lib, heads=1 << 12, page=1 << 12, D=256) == -2
    # nothing to do
    assert attend(lib, B=0) == 0 and append(lib, B=0) == 0 and extend(lib, B=0) == 0 and truncate(lib, B=0) == 0
    assert fork(lib, forks=0) == 0 and copy(lib, n=0) == 0


def test_the_binding_refuses_what_it_cannot_hand_over():
    c = cp.make(2, 3, 4, 2, 8, 4, [5, 6], device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens)
    with pytest.raises(ValueError, match="CUDA"):
        bv.bv_pages_extend(c.table, c.lens, c.refs, 4, 1)
    with pytest.raises(ValueError, match="int32"):
        bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, c.table.long(), c.lens)
    with pytest.raises(ValueError, match="contiguous"):
        bv.bv_pages_truncate(c.table.t().contiguous().t(), c.lens, c.refs, 4, c.lens)
    with pytest.raises(ValueError, match="rows of D"):
        bv.bv_cache_attend(c.q, c.k.transpose(2, 3), c.v, c.table, c.lens)


def test_the_plain_bookkeeping():
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)                                         # noqa: E731
    b = cp.Book(i32([[0, 1, -1], [0, 1, -1], [3, -1, -1]]), i32([6, 6, 4]), i32([2, 2, 0, 1, 0, 0]), 4)
    assert b.extend(3, [3, 0, 1]) == ([3, 0, 1], [[1, 2], [-1, -1], [-1, -1]])               # page 1 is shared: 2 in its place, 4 behind it; 5 for the third
    assert b.table == [[0, 2, 4], [0, 1, -1], [3, 5, -1]] and b.lens == [9, 6, 5] and b.refs == [2, 1, 1, 1, 1, 1]
    b.truncate([1, 9, 0], 3, [3, 0, 1])
    assert b.lens == [7, 6, 4] and b.table == [[0, 2, -1], [0, 1, -1], [3, -1, -1]] and b.refs == [2, 1, 1, 1, 0, 0]
    assert b.fork([0, 1, 2], [2, 2, 0]) == [-1, -1, -1]                                      # 2 twice; 0 is a source
    assert b.fork([0], [2]) == [0] and b.lens == [7, 6, 7] and b.refs == [3, 1, 2, 0, 0, 0]
    b.truncate([0, 6, 0])
    assert b.refs == [1, 1, 0, 0, 0, 0]
    b.refs = [0, 1, 0, 1, 0, 0]
    b.table[1] = [3, 1, -1]
    assert b.compact() == ([[3, 0], [-1, -1], [-1, -1]], 1) and b.table[1] == [0, 1, -1] and b.refs == [1, 1, 0, 0, 0, 0]


def test_the_plain_attention_on_a_case_by_hand():
    """Two keys with scores 0 and ln 3, values 1 and 5: (1 + 3 * 5) / 4 = 4; the window of one sees the second alone."""
    k = torch.zeros((1, 1, 2, 8))
    v = torch.zeros((1, 1, 2, 8))
    k[0, 0, 1, 0] = torch.tensor(3.0).log()
    v[0, 0, 0], v[0, 0, 1] = 1.0, 5.0
    q = torch.zeros((1, 1, 1, 8))
    q[..., 0] = 1.0
    table, lens = torch.zeros((1, 1), dtype=torch.int32), torch.tensor([2], dtype=torch.int32)
    out, bound, written = cp.attend(q, k, v, table, lens, scale=1.0)
    assert (out - 4).abs().max() < 1e-7 and written.all() and 0 < bound.max() < 1e-4
    assert (cp.attend(q, k, v, table, lens, scale=1.0, window=1)[0] == 5).all()
    assert ((cp.attend(q, k, v, table, lens, scale=1.0, window=1, sinks=1)[0] - 4).abs() < 1e-7).all()


# ---- what the kernels are handed, over the runtime of tests/host_runtime.cu ----

@pytest.fixture(scope="module")
def host_so(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    built = bv_build.build()
    out = str(tmp_path_factory.mktemp("host") / "host_cache.so")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17",
                           "-Xcompiler", "-fPIC", "-shared", "-I", bv_build.CSRC, os.path.join(here, "host_cache.cu"), "-o", out,
                           "-Xlinker", "-Bsymbolic", "-Xlinker", "-rpath=" + os.path.dirname(built), built])
    return ctypes.CDLL(out)


@pytest.fixture
def host(host_so):
    host_so.bv_release()
    host_so.host_errors.restype = ctypes.c_char_p
    host_so.host_live_bytes.restype = ctypes.c_size_t
    yield host_so
    host_so.host_refuse_tiles(0)
    host_so.bv_release()


def on_host(host, B=3, n=1, q_heads=8, heads=2, D=128, page=16, dtype=1, offset=0, stream=None):
    status = host.host_attend(B, n, q_heads, heads, D, page, dtype, ctypes.c_longlong(offset), ctypes.c_void_p(stream))
    return status, host.host_attend_kernel()


def test_the_parts_fit_the_workspace_whatever_the_shape(host):
    for dtype in (0, 1):
        for D in (8, 33, 64, 80, 128, 136, 256):
            for n in (1, 2, 9, 17, 300):
                for group in (1, 3, 8, 64):
                    for page in (1, 16, 24, 200):
                        assert on_host(host, n=n, q_heads=2 * group, D=D, page=page, dtype=dtype)[0] == 0
                        assert host.host_errors() == b"", (dtype, D, n, group, page)


def test_which_kernel_takes_a_call(host):
    assert on_host(host)[1] == 1                                        # bf16 in whole vectors: the tensor cores
    assert on_host(host, dtype=0)[1] == 2                               # 32 bits
    assert on_host(host, offset=1)[1] == 2 and on_host(host, D=36)[1] == 2 and on_host(host, D=136)[1] == 2 and on_host(host, page=20)[1] == 2
    assert on_host(host, D=72, page=24)[1] == 1 and on_host(host, D=16, page=8)[1] == 1 and on_host(host, page=1000)[1] == 1
    host.host_refuse_tiles(1)                                           # no map of the pools: the other kernels, planned anew
    for n in (1, 5, 40):
        assert on_host(host, n=n) == (0, 2) and host.host_errors() == b""
    host.host_refuse_tiles(0)
    # rows of a unit: as even as multiples of 16 are, no more units than have to be
    for rows, want in ((1, 16), (16, 16), (17, 32), (72, 80), (80, 80), (81, 48), (136, 80), (161, 64), (272, 80)):
        on_host(host, n=rows, q_heads=1, heads=1)
        assert host.host_attend_rows() == want, rows


def test_calls_of_several_sizes_and_their_replays_share_a_workspace(host):
    sizes = [dict(), dict(n=9, q_heads=64, heads=8), dict(n=300, q_heads=8), dict(dtype=0, n=5, q_heads=10, D=80, page=24)]
    for a in sizes:
        for b in sizes:
            host.bv_release()
            on_host(host)                                               # (the library is set up before any capture)
            host.host_begin_capture(None)
            assert on_host(host, **a)[0] == 0
            graph = host.host_end_capture()
            for step in (b, None, b, a, None, None, b):
                host.host_replay(graph) if step is None else on_host(host, **step)
                assert host.host_errors() == b"", (a, b)
    host.bv_release()
    assert host.host_live_bytes() == 0 and host.host_errors() == b""
