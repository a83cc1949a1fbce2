"""LayerOps' own checks, without a GPU."""
import pytest
import torch

from paper_2403_16125_amd import arena, layer


@pytest.fixture
def ops():
    o = layer.LayerOps()
    yield o
    o.close()


@pytest.mark.parametrize("typ", [torch.float64, torch.int32, torch.float8_e4m3fn])
def test_types_that_no_norm_takes(ops, typ):
    """Of the stream, of the block's output, or asked for: each is named."""
    x, odd = torch.zeros(2, 8), torch.zeros(2, 8).to(typ)
    none = (None, 0, 1.0, None, None, None, None, "rms", 1e-6)
    for args in ((odd, None, *none, None, True, False), (x, odd, *none, None, True, False),
                 (x, None, *none, typ, True, False)):
        with pytest.raises(ValueError, match=f"type {typ} is not supported"):
            ops._norm_forward(0, *args)
    stats = torch.zeros(2, 4)
    for args in ((x, x, odd, x, stats), (odd, x, x, None, stats), (x, x, x, odd, stats)):
        with pytest.raises(ValueError, match=f"type {typ} is not supported"):
            ops._norm_backward(0, *args, *none)


def test_calls_after_close_are_refused():
    """The context is gone: nothing is handed to the library, whatever the call."""
    o = layer.LayerOps()
    o.close()
    assert o.ctx is None
    with pytest.raises(arena.ArenaError) as e:
        layer.arena_norm_forward(o.ctx, layer.NormDesc())
    assert e.value.status == 1
    for query in (lambda: layer.arena_ffn_forward_workspace(o.ctx, layer.FfnDesc()),
                  lambda: layer.arena_orthogonal_update_workspace(o.ctx, layer.UpdateDesc())):
        with pytest.raises(arena.ArenaError):
            query()
    o.close()
