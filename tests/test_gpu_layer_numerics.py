"""What the layer operators round, and where: cases beside Gaussian inputs and
dense calls."""
import pytest
import torch

import layer_reference as ref
from paper_2403_16125_amd import layer

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
CODES = {F32: 0, BF16: 1, F16: 2}


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def normal(shape, dtype, seed, std=1.0, mean=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T,D,rows", [(37, 9000, 7), (300, 8195, 0), (5, 16384, 2), (40, 8192, 9), (33, 700, 5)])
def test_norm_backward_in_place_gives_the_same_bits(ops, T, D, rows, typ, kind):
    """dx over dr with a 16-bit stream: the gradient of r is rounded as it is stored,
    and the sums of gates, weights and biases come from it unrounded all the same."""
    groups = -(-T // rows) if rows else 1
    x, y, dr = normal((T, D), typ, 1, 2.0), normal((T, D), typ, 2, 0.7, 0.1), normal((T, D), typ, 3, 0.3)
    dn, gate = normal((T, D), typ, 4, 0.3), normal((groups, D), typ, 5, 0.3, 0.5)
    w2, w1, b2, b1 = (normal((D,), typ, 6 + i, 0.1, 1.0) for i in range(4))
    given = dict(gate=gate, gate_rows=rows, scale=0.5, w_post=w2, w_pre=w1, kind=kind)
    if kind == "layer":
        given.update(b_post=b2, b_pre=b1)
    r, n, stats = ops.norm_forward(x, y, save=True, **given)
    want = ops.norm_backward(dn, dr, r, y, stats, **given)
    p = lambda t: None if t is None else t.data_ptr()
    d = layer.NormDesc(dtype=CODES[typ], stream_dtype=CODES[typ], kind=layer.NORM_KINDS[kind], width=D, tokens=T,
                       gate_rows=rows, eps=1e-6, scale=0.5, y=p(y), ld_y=D, gate=p(gate), ld_gate=D, w_post=p(w2),
                       b_post=p(given.get("b_post")), w_pre=p(w1), b_pre=p(given.get("b_pre")), r=p(r), ld_r=D,
                       stats=p(stats))
    need = layer.arena_norm_backward_workspace(ops.ctx, d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    got = {k: torch.empty_like(v) for k, v in want.items() if v is not None}
    got["dx"] = dr.clone()
    g = layer.NormGrads(dn=p(dn), ld_dn=D, dr=p(got["dx"]), ld_dr=D, dx=p(got["dx"]), ld_dx=D, dy=p(got["dy"]), ld_dy=D,
                        workspace=p(ws), workspace_bytes=need, **{k: p(v) for k, v in got.items() if k not in ("dx", "dy")})
    layer.arena_norm_backward(ops.ctx, d, g, torch.cuda.current_stream().cuda_stream)
    for k in got:
        assert torch.equal(got[k], want[k]), k
