"""Rotary positions: outputs that cannot hold what the call writes."""
import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_outputs_that_lie_on_each_other():
    """Expanded tensors are read as what they stand for, and refused as outputs, in place as well."""
    r, pos = binding.Rope(64), torch.arange(5, dtype=torch.int32, device=DEV)
    one = torch.randn(1, 2, 64, device=DEV)
    x = one.expand(5, 2, 64)
    assert torch.equal(r.apply(pos, x), r.apply(pos, x.contiguous()))
    for out in (x, torch.zeros(5, 1, 64, device=DEV).expand(5, 2, 64)):
        with pytest.raises(ValueError, match="on each other"):
            r.apply(pos, x, q_out=out)
    k = torch.randn(5, 2, 64, device=DEV)
    with pytest.raises(ValueError, match="on each other"):
        r.apply(pos, k, k, q_out=torch.empty_like(k), k_out=x)
    single = torch.randn(1, 1, 64, device=DEV)
    out = torch.zeros(64, device=DEV).as_strided((1, 1, 64), (0, 0, 1))       # (axes of one: nothing lies on anything)
    assert r.apply(pos[:1], single, q_out=out) is out and torch.equal(out, single)
