"""Arithmetic that the cache's kernels share with the host, at the ends of its ranges."""
import ctypes
import itertools
import os
import random
import subprocess
import sys

import pytest

from paper_2403_10444_b200 import build as bv_build

MOST = 2**31 - 1024


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    out = str(tmp_path_factory.mktemp("host") / "host_arithmetic.so")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-Xcompiler", "-fPIC",
                           "-shared", "-I", bv_build.CSRC, os.path.join(here, "host_arithmetic.cu"), "-o", out])
    return ctypes.CDLL(out)


def test_a_token_is_stored_inside_its_sequence_or_nowhere(host):
    """Lengths that are none, down to the lowest integer (one less than which is the largest), have no places."""
    for (width, page), m in itertools.product(((3, 16), (1, 1), (1 << 22, 1 << 20), (100, 16)), (-2**31, -1, 0, 1, 2, 17, 2**30, 2**31 - 1)):
        ends = (-2**31, -2**31 + 1, -2**31 + 16, -17, -1, 0, 1, 2, 16, 17, width * page, width * page + 1, MOST, MOST + 1, 2**31 - 1)
        for length in {x for x in ends if -2**31 <= x < 2**31}:
            for t in {0, 1, 16, max(0, m - 1), max(0, m)}:
                if t >= 2**31:
                    continue
                fits = 0 <= length <= min(MOST, width * page) and t < m
                want = length - m + t if fits and length - m + t >= 0 else None
                got = host.host_place_of(length, m, t, width, page)
                assert got == want if want is not None else got < 0, (length, m, t, width, page)


def test_sums_of_pages_that_many_sequences_ask_for(host):
    """In rounds of 512 sequences, as extending adds them up: never below what came before, never beyond a page more than there are."""
    most = 2**22 - 2
    for P in (1, 100, most - 9000, most):
        for want in (0, 1, P // 2, P, P + 1):
            carry = true = 0
            for _ in range(16):
                for i in (1, 2, 511, 512):
                    assert host.host_sum_up_to(P + 1, carry, i * want) == min(true + i * want, P + 1), (P, want)
                carry, true = host.host_sum_up_to(P + 1, carry, 512 * want), true + 512 * want


def test_rows_of_as_many_bytes_as_32_bits_hold_and_more():
    """Up to the launch, in a process of its own (a division by zero ends it); without a device the launch is what fails."""
    code = ("import sys; sys.path[:0] = %r\n"
            "import test_cache_cpu as t\n"
            "from paper_2403_10444_b200 import build, binding\n"
            "build.build(); lib = binding.load_library()\n"
            "for D in (2**29, 2**30, 2**31 - 4, 2**31 - 1):\n"
            "    for dtype in (0, 1):\n"
            "        assert t.append(lib, D=D, B=0, dtype=dtype) == 0\n"
            "        if not t.torch.cuda.is_available():\n"
            "            assert t.append(lib, D=D, dtype=dtype) == -3\n"
            "            assert t.copy(lib, D=D, heads=1, page=1, dtype=dtype) == (-3 if D < 2**30 else -2)\n")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.check_call([sys.executable, "-c", code % [os.path.dirname(here), here]])


def test_divisions_by_what_the_host_knows(host):
    """Quotients of everything below 2^31 at which they could differ: multiples of the divisor and their neighbours, the ends."""
    rng = random.Random(1)
    divisors = [1, 2, 3, 5, 7, 16, 24, 48, 127, 128, 641, 2**20, 2**30 - 1, 2**30, 2**30 + 1, 2**31 - 2, 2**31 - 1] + [rng.randrange(1, 2**rng.randint(1, 31)) for _ in range(300)]
    for by in divisors:
        top = (2**31 - 1) // by
        near = {0, 1, top, max(0, top - 1), top // 2} | {rng.randint(0, top) for _ in range(20)}
        for n in {q * by + d for q in near for d in (-1, 0, 1, by - 1)} | {2**31 - 1}:
            if 0 <= n < 2**31:
                assert host.host_divide(by, n) == n // by, (by, n)
