"""The binding of the operators of a layer of experts refuses sizes that a descriptor's
fields would cut off, without a GPU: tensors of the meta device have any size and no memory."""
import pytest
import torch

from paper_2403_16125_amd import layer
from paper_2403_16125_amd import layer_experts as le

I32, F32 = torch.int32, torch.float32


@pytest.fixture
def ops():
    o = layer.LayerOps()
    o._index, o.dev = -1, torch.device("meta")      # of tensors without memory
    yield o
    o.close()


def some(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("k", [2 ** 31, 2 ** 32 + 2])
def test_choices_that_a_field_would_cut_off(ops, k):
    """2^32 + 2 choices a token would be taken as 2, the rest of the rows left unwritten."""
    row = some(1, k, dtype=I32)
    plan = le.ExpertPlan(some(9, dtype=I32), row)
    x, ys = some(1, 8), some(k, 8)
    for call in (lambda: ops._sort_by_expert(0, row, 8), lambda: ops._dispatch(0, x, plan, ys),
                 lambda: ops._combine(0, ys, plan, None, x), lambda: ops._combine_backward(0, x, ys, plan, some(1, k), ys),
                 lambda: ops._route_backward(0, some(1, k), some(1, 8), row, True, 1.0)):
        with pytest.raises(ValueError, match=f"has {k} choices a token"):
            call()


@pytest.mark.parametrize("experts", [2 ** 31, 2 ** 32 + 1])
def test_experts_that_a_field_would_cut_off(ops, experts):
    w = some(experts, 1, 1, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=f"has {experts} experts"):
        ops._experts_forward(0, some(4, 1, dtype=torch.bfloat16), some(experts + 1, dtype=I32), w, w, w, "silu", False, None)
