"""Nucleus cuts whose border lies where tokens are many and light, or where distances leave the range of 32 bits, against sums in 64 bits."""
import math

import pytest
import torch

import paper_2403_10444_b200 as bv
from test_gpu_filter import check, uniforms

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("V,bits,p,top_k", [(1 << 22, 41, 1 - 2.0 ** -20, 0), (1 << 22, 41, 1 - 2.0 ** -20, 3 << 20), (128256, 40, 1 - 2.0 ** -24, 0), (1 << 26, 37, 1 - 2.0 ** -12, 0)])
def test_a_nucleus_of_light_tokens(V, bits, p, top_k):
    """One token, and V - 1 of some 2^-bits of its weight which hold the border: about half of them are kept.

    Beside the first token's 1 sums in 64 bits are good to some 2^-52 an addition; what is light is summed up exactly to 2^-69, V times: 2^-43 in all, less than half a
    token of 2^-41, so at most one token more or less than the border has."""
    assert float(torch.tensor(p, dtype=F32)) == p
    gen = torch.Generator(device="cuda").manual_seed(V + top_k)
    z = torch.rand((1, V), device="cuda", generator=gen) * -0.007 - bits * math.log(2)
    z[0, V // 3] = 0.0
    u = torch.tensor([1 - 2.0 ** -24], device="cuda")
    out = torch.empty_like(z)
    bv.bv_sample_filtered(z, u, top_p=p, top_k=top_k, out_logits=out)
    order = z[0].sort(descending=True, stable=True).indices[:top_k or V]
    w = z[0, order[1:]].double().exp()
    before = w.cumsum(0) - w
    # the first token weighs 1: 1 + before < p (1 + sum)
    want = 1 + int((before < p * w.sum() - (1 - p)).sum())
    kept = out[0] > -math.inf
    n = int(kept.sum())
    assert V // 8 < want < V - V // 8 and abs(n - want) <= 1, (n, want)
    first = torch.zeros_like(kept)
    first[order[:n]] = True
    assert torch.equal(kept, first) and torch.equal(out[0][kept], z[0][kept])


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
