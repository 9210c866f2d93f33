"""Calls of the cut rows that are refused before anything is written."""
import pytest
import torch

import paper_2403_10444_b200 as bv
from paper_2403_10444_b200 import binding
from test_gpu_filter import rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fast", [True, False])
def test_no_uniforms(monkeypatch, fast):
    if not fast:
        monkeypatch.setattr(binding, "_fast", None)
    z = rows_of(3, 100, torch.float32, "wide")
    out = torch.full_like(z, 5.0)
    with pytest.raises(ValueError):
        bv.bv_sample_filtered(z, None, top_k=3, out_logits=out)
    torch.cuda.synchronize()
    assert bool((out == 5.0).all())
