"""The ends of the uniforms' range on cut rows: 0 is the first kept token that weighs anything, whatever was cut before it; and what is drawn is always kept."""
import pytest
import torch

import paper_2403_10444_b200 as bv
import prompt_plain as pp
from test_gpu_filter import rows_of

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CUTS = [dict(), dict(top_k=1), dict(top_k=3), dict(top_k=300, top_p=0.99), dict(top_p=0.5), dict(top_p=0.97), dict(min_p=0.2), dict(top_k=40, temperature=0.02), dict(top_k=1500, min_p=0.001)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("law", ["zipf", "wide", "steps", "masked", "equal"])
@pytest.mark.parametrize("rows,V", [(3, 37), (3, 1999), (2, 5003), (1, 32000), (160, 4097)])
def test_the_ends(rows, V, law, dtype):
    z = rows_of(rows, V, dtype, law, seed=V)
    for u in (0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24):
        for cut in CUTS:
            tokens, _ = bv.bv_sample_filtered(z, torch.full((rows,), u, device="cuda"), **cut)
            for r in range(0, rows, 40):
                kept, w = pp.cut(z[r], cut.get("temperature", 1.0), cut.get("top_k", 0), cut.get("top_p", 1.0), cut.get("min_p", 0.0))
                token = tokens[r].item()
                assert bool(kept[token]) and w[token] > 0, (u, cut)
                # (sums of V weights, in whatever order, are off by some 10^-11 of them at most)
                upto = w.cumsum(0)
                assert upto[token] - w[token] <= (u + 1e-11) * upto[-1] and upto[token] >= (u - 1e-11) * upto[-1], (u, cut)
                if u == 0.0:
                    assert token == int((w > 0).to(torch.int32).argmax()), cut
