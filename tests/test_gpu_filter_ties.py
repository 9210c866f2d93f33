"""Cuts by number and by mass together where many tokens are equal: the mass keeps none that the number has cut."""
import pytest
import torch

from test_gpu_filter import check, rows_of, uniforms

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("law", ["equal", "steps", "large"])
@pytest.mark.parametrize("rows,V", [(2, 8192), (1, 50257), (150, 5003)])
def test_a_mass_that_takes_all_of_the_number(rows, V, law, dtype):
    z = rows_of(rows, V, dtype, "equal" if law == "large" else law)
    if law == "large":
        z.fill_(1e30)
    # (10^30 at a temperature of 10^-30 has a normaliser that 32 bits do not hold)
    cold = 1e-30 if law != "large" else 1e-6
    for cut in (dict(top_k=4873), dict(top_k=4999, min_p=0.05), dict(top_k=2, temperature=3e37), dict(top_k=200, temperature=3e37), dict(top_k=1030, temperature=cold)):
        for p in (0.999999, 0.5):
            check(z[:3], uniforms(min(rows, 3)), top_p=p, **cut)
            if rows > 3:
                check(z, uniforms(rows), top_p=p, **cut)
