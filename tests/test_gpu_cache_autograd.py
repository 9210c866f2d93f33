"""The cache's calls are forward only, as they say: with tensors that require gradients they do the same, and leave no graph."""
import pytest
import torch

import cache_plain as cp
import paper_2403_10444_b200 as bv
from paper_2403_10444_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("way", ["fast", "interpreted"])
@pytest.mark.parametrize("some", [False, True])
def test_no_graph(way, some, monkeypatch):
    if way == "interpreted":
        monkeypatch.setattr(binding, "_fast", None)
    c = cp.make(3, 2, 4, 2, 64, 16, [40, 3, 100])
    new = torch.tensor([2, 1, 0], dtype=torch.int32, device="cuda") if some else None
    want = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, n_new=new)
    for t in (c.q, c.k, c.v, c.k_new, c.v_new):
        t.requires_grad_(True)
    got = bv.bv_cache_attend(c.q, c.k, c.v, c.table, c.lens, n_new=new)
    assert torch.equal(got, want) and not got.requires_grad and got.grad_fn is None
    bv.bv_cache_append(c.k_new, c.v_new, c.k, c.v, c.table, c.lens, n_new=new)
    assert c.k.grad_fn is None and c.v.grad_fn is None
    with torch.no_grad():
        assert torch.equal(c.k[c.table[0, 38 // 16].item(), :, 38 % 16], c.k_new[0, 0])
    assert "orward only" in bv.bv_cache_attend.__doc__
