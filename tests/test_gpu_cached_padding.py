"""Prompts of different lengths in one batch of the decoding loop on the cache: what lies beyond a prompt does not matter."""
import pytest
import torch

from paper_2403_10444_b200 import cached
from test_gpu_cached_loop import setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_lies_beyond_a_prompt_is_not_looked_at(dtype):
    tw, dw, prompts, lens, ud, uv, make = setup(dtype, head_dim=64)
    want = cached.run(*make(), prompts, lens, ud, uv, 3)
    for pad in (-1, 512, 2**31 - 1, -2**31):
        beyond = torch.arange(prompts.shape[1], device="cuda")[None, :] >= lens[:, None]
        got = cached.run(*make(), torch.where(beyond, torch.full_like(prompts, pad), prompts), lens, ud, uv, 3)
        assert all(torch.equal(want[k], got[k]) for k in want)
