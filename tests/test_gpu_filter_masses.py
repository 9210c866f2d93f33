"""Nucleus cuts whose distances leave the range of 32 bits, against sums in 64 bits."""
import pytest
import torch

from test_gpu_filter import check, uniforms

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V", [(3, 2500), (1, 40000)])
def test_distances_beyond_the_range(dtype, rows, V):
    """Logits of both ends of the type at a temperature of their size: weights of e^-6 at a distance that 32 bits do not hold."""
    gen = torch.Generator().manual_seed(V)
    z = -2.9e38 - torch.rand((rows, V), generator=gen) * 1e37
    z[:, V // 2] = 3e38
    z = z.to(dtype).cuda()
    for cut in (dict(top_p=0.9), dict(top_p=0.5, top_k=2100), dict(top_p=0.7, min_p=0.001)):
        check(z, uniforms(rows), temperature=1e38, **cut)
    # (and at an ordinary temperature the first one is all there is)
    check(z, uniforms(rows), top_p=0.9)
