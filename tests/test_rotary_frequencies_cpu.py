"""Frequencies for stretched contexts, by values worked out beside the formulas."""
import math

import torch

import paper_2403_10444_b200 as bv


def test_by_parts():
    # 64 elements, base 10^4: pair i turns 10^(-i / 8) a position, so over 2048 positions 326 10^(-i / 8) times.  32 turns are at i = 8.06, one at i = 20.1: pairs up to 8 stay as
    # they are, those from 21 on turn an eighth as fast, between them a ramp of 13 steps
    f = bv.rotary_frequencies(64, 10000.0, factor=8.0, original=2048, device="cpu")
    assert f.shape == (32,) and f.dtype == torch.float64
    for i, share in ((0, 0.0), (8, 0.0), (9, 1 / 13), (14, 6 / 13), (20, 12 / 13), (21, 1.0), (31, 1.0)):
        plain = 10.0 ** (-i / 8)
        assert math.isclose(f[i].item(), plain * (1 - share) + plain / 8 * share, rel_tol=1e-14), i


def test_by_parts_with_bounds_of_ones_own():
    # base 16, eight elements: pair i turns 2^-i a position, over 64 pi positions (201, to a whole number) 32 2^-i times but for some 10^-3.  Eight turns are next to i = 2, four next to 3
    f = bv.rotary_frequencies(8, 16.0, factor=2.0, original=201, low=3.9, high=8.1, device="cpu")
    # last index with 8.1 turns or more: 1; first with 3.9 or fewer: 4
    want = [1.0, 0.5, 0.25 * (2 / 3 + 1 / 6), 0.125 * (1 / 3 + 2 / 6)]
    assert all(math.isclose(a, b, rel_tol=1e-14) for a, b in zip(f.tolist(), want))


def test_a_context_in_which_all_turn_often():
    plain = bv.rotary_frequencies(8, device="cpu")
    assert torch.equal(bv.rotary_frequencies(8, factor=4.0, original=10**9, device="cpu"), plain)
