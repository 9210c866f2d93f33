"""Units of the prompts' kernel that follow one another on a CTA: what one leaves behind does not reach the next."""
import math

import pytest
import torch

import paper_2403_10444_b200 as bv
from test_gpu_prompt import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("lens,Hq,Hkv,D", [([200, 300] + [50] * 400, 16, 16, 64), ([260] * 3 + [20, 7, 128] * 100, 8, 8, 128)])
def test_values_that_are_not_finite_in_units_of_one_tile(lens, Hq, Hkv, D, value):
    """Thousands of units without a second tile behind some that have one; every seventh sequence has a value that is not finite, which its later rows see."""
    q, k, v, off = make(lens, Hq, Hkv, D, tail=2)
    clean = check(q, k, v, off)
    bad, want = v.clone(), clean.clone()
    for b in range(0, len(lens), 7):
        first, end = off[b].item(), off[b + 1].item()
        at, h = first + min(5, end - first - 1), b % Hkv
        bad[at, h, 3] = value
        want[at:end, h, 3] = value
    for _ in range(5):
        got = torch.full_like(clean, 3.0)
        bv.bv_prompt_attend(q, k, bad, off, out=got)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (14, 2), (65, 1)])
def test_other_prompts_queries_and_what_ran_before_change_no_bit(Hq, Hkv, D):
    """Rows of a tile that are nobody's hold another prompt's queries, or (where the group does not divide 128) what earlier calls left: large ones, not finite ones."""
    lens = [45, 60, 3, 130]
    q, k, v, off = make(lens, Hq, Hkv, D, seed=D + Hq)
    want = check(q, k, v, off)
    before = make([128 * 40], 4, 4, D, seed=1)
    for size in (1e5, 1e20, math.inf, math.nan):
        for b in (1, 3):
            other = q.clone()
            other[off[b]:off[b + 1]] *= size
            got = bv.bv_prompt_attend(other, k, v, off)
            mine = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
            mine[off[b]:off[b + 1]] = False
            assert torch.equal(got[mine], want[mine]), (size, b)
        large = before[0].clone().mul_(size)
        for _ in range(3):
            bv.bv_prompt_attend(large, *before[1:])
            assert torch.equal(bv.bv_prompt_attend(q, k, v, off), want), size
