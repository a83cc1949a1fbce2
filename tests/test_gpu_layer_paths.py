"""The layer operators on the GPU at shapes that take every path through the tiled
products (test_layer_paths.py), large ones among them, against 64 bits.

Feed-forward: the elementwise bounds of layer_reference, and 2 u of each result's
norm: one rounding of its own and independent ones of the operands of its products, at
most u each (the elementwise bounds grow with the sums' lengths and would pass a
step of k left out).  Update: three steps, 1e-2 of the norm over all, and 3e-2 of the
same size in each of 16 x 16 parts of a matrix, which one tile left out would pass."""
import pytest
import torch

import layer_reference as ref
from layer_launches import SHAPES
from paper_2403_16125_amd import layer

pytestmark = pytest.mark.gpu

TYPES = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}
ACTS = ("silu", "gelu", "relu")


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def normal(shape, dtype, seed, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def near(name, got, want, bound, u):
    off = got.double().sub_(want)
    assert off.norm() <= 2 * u * want.norm(), f"{name}: {(off.norm() / want.norm()).item()}"
    assert bool((off.abs_() <= bound).all()), name


@pytest.mark.parametrize("typ,act,T,D,F,grad,accumulate", [s[1:] for s in SHAPES if s[0] == "ffn"])
def test_ffn_paths(ops, typ, act, T, D, F, grad, accumulate):
    typ, act, grad = TYPES[typ], ACTS[act], TYPES[grad]
    x, wg, wu = normal((T, D), typ, 1), normal((F, D), typ, 2, D ** -0.5), normal((F, D), typ, 3, D ** -0.5)
    wd, dy = normal((D, F), typ, 4, F ** -0.5), normal((T, D), typ, 5, 0.25)
    y, saved = ops.ffn_forward(x, wg, wu, wd, activation=act, save=True)
    want, bound, kept = ref.ffn(x, wg, wu, wd, act, typ)
    near("y", y, want, bound, ref.U[typ])
    grads = [normal(w.shape, grad, 6 + i) if accumulate else torch.empty(w.shape, dtype=grad, device="cuda")
             for i, w in enumerate((wg, wu, wd))]
    before = [g.double() for g in grads] if accumulate else [None] * 3
    got = ops.ffn_backward(dy, x, wg, wu, wd, saved, activation=act, grads=grads, accumulate=bool(accumulate))
    back = ref.ffn_back(dy, x, wg, wu, wd, act, typ, kept, grad)
    for (name, (v, b)), g, add in zip(back.items(), got, (None, *before)):
        if add is not None:
            b = b + ref.U[grad] * (v.abs() + add.abs())
            v = v + add
        near(name, g, v, b, ref.U[typ])


@pytest.mark.parametrize("typ,batch,rows,cols", [s[1:] for s in SHAPES if s[0] == "update"])
def test_update_paths(ops, typ, batch, rows, cols):
    grad = normal((batch, rows, cols), TYPES[typ], 1, 0.01)
    got = ops.orthogonal_update(grad, steps=3)
    r, c = -(-rows // 16), -(-cols // 16)
    for g, v in zip(got, grad):
        want = ref.orthogonal(v, layer.COEFFICIENTS, 3, 1e-7, 1.0)
        off = g.double() - want
        assert off.norm() <= 1e-2 * want.norm()
        parts = torch.zeros(16 * r, 16 * c, dtype=torch.float64, device="cuda")
        parts[:rows, :cols] = off
        parts = (parts ** 2).view(16, r, 16, c).sum((1, 3))
        assert bool((parts <= r * c * (3e-2 * want.norm()) ** 2 / (rows * cols)).all())


@pytest.mark.parametrize("typ", [1, 2])
@pytest.mark.parametrize("T,D,F", [(1, 4104, 700), (16, 5001, 333), (20, 4100, 1001), (32, 6144, 1360), (1, 2048, 4100),
                                   (31, 700, 9001)])
def test_few_tokens_of_wide_blocks(ops, typ, T, D, F):
    """Up to 32 tokens: more than 4096 columns of the model take half as many waves a block."""
    typ = TYPES[typ]
    x, wg, wu = normal((T, D), typ, 1), normal((F, D), typ, 2, D ** -0.5), normal((F, D), typ, 3, D ** -0.5)
    wd = normal((D, F), typ, 4, F ** -0.5)
    y = ops.ffn_forward(x, wg, wu, wd, activation="gelu")
    want, bound, _ = ref.ffn(x, wg, wu, wd, "gelu", typ)
    near("y", y, want, bound, ref.U[typ])
