"""The experts' blocks and the loss on the GPU at shapes that take every path through the
products of groups and of a loss (test_expert_paths.py), large ones among them, against 64 bits:
the elementwise bounds of layer_reference and experts_reference, and of each
result's norm 2 u: one rounding of its own and independent ones of the operands of its
products, at most u each (the elementwise bounds grow with the sums' lengths and would pass a
step of k left out).

ReLU's derivative jumps by 1 where g is 0, so where g is nearer to 0 than its sum's rounding
either side is right: a gradient of 2048 x 192 whose norm is 2572 has rows of |dg| |x| = 0.2 x 14 that
one such g adds or leaves out, 1.1e-3 of the norm, more than 2 u in float16.  There the formulas take the side of the g
that the forward pass kept, and everywhere else that has to be the formulas' own."""
import pytest
import torch

import experts_reference as exp
import layer_reference as ref
from expert_launches import SHAPES, counts
from paper_2403_16125_amd import layer
from test_gpu_layer_paths import ACTS, TYPES, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def near(name, got, want, bound, u):
    """A result below its type's normal numbers is off by up to half of the least subnormal (2^-25 in float16, where
    dx of a mean over 5702 tokens is 1e-7 to 3e-5: in 12.8 million values 1.1e-4 of a norm of 0.0385)."""
    off = got.double().sub_(want)
    least = 0.5 * ref.TINY[got.dtype] * got.numel() ** 0.5
    assert off.norm() <= 2 * u * want.norm() + least, f"{name}: {(off.norm() / want.norm()).item()}"
    assert bool((off.abs_() <= bound).all()), name


def kept_g(saved, inner):
    """g as the forward pass kept it: 16-bit heads of all rows, then their 8-bit tails."""
    _, at, _, _ = saved.parts()
    n = saved.tokens * saved.ld
    head = saved.buffer[at:at + 2 * n].view(torch.int16).view(saved.tokens, saved.ld)[:, :inner].int() << 16
    tail = saved.buffer[at + 2 * n:at + 3 * n].view(saved.tokens, saved.ld)[:, :inner].int() << 8
    return (head | tail).view(torch.float32)


def gradient(shape, typ, accumulate, seed):
    """A buffer for a gradient, and what it holds that is added to."""
    g = normal(shape, typ, seed) if accumulate else torch.empty(shape, dtype=typ, device="cuda")
    return g, g.clone() if accumulate else None


def added(v, bound, before, typ):
    if before is None:
        return v, bound
    return v + before.double(), bound + ref.U[typ] * (v.abs() + before.double().abs())


@pytest.mark.parametrize("typ,act,rows,D,F,E,grad,accumulate", [s[1:] for s in SHAPES if s[0] == "experts"])
def test_experts_paths(ops, typ, act, rows, D, F, E, grad, accumulate):
    typ, act, grad = TYPES[typ], ACTS[act], TYPES[grad]
    bounds = [0]
    for n in counts(rows, E):
        bounds.append(bounds[-1] + n)
    offsets = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    x, dy = normal((rows, D), typ, 1), normal((rows, D), typ, 5, 0.25)
    wg, wu = normal((E, F, D), typ, 2, D ** -0.5), normal((E, F, D), typ, 3, D ** -0.5)
    wd = normal((E, D, F), typ, 4, F ** -0.5)
    ys, saved = ops.experts_forward(x, offsets, wg, wu, wd, activation=act, save=True)
    grads, before = zip(*(gradient(w.shape, grad, accumulate, 6 + i) for i, w in enumerate((wg, wu, wd))))
    dx, *dw = ops.experts_backward(dy, x, offsets, wg, wu, wd, saved, activation=act, grads=grads,
                                   accumulate=bool(accumulate))
    g_kept = kept_g(saved, F) if act == "relu" else None
    for e in range(E):
        at = slice(bounds[e], bounds[e + 1])
        if bounds[e] == bounds[e + 1]:
            assert all(torch.equal(g[e], b[e]) if accumulate else not g[e].any() for g, b in zip(dw, before))
            continue
        want, bound, kept = ref.ffn(x[at], wg[e], wu[e], wd[e], act, typ)
        near(f"ys of {e}", ys[at], want, bound, ref.U[typ])
        if act == "relu":
            own = g_kept[at].double()
            open_ = kept["g"].abs() <= kept["bg"]
            assert bool((open_ | ((own > 0) == (kept["g"] > 0))).all())
            kept["g"] = torch.where(open_, own, kept["g"])
        back = ref.ffn_back(dy[at], x[at], wg[e], wu[e], wd[e], act, typ, kept, grad)
        near(f"dx of {e}", dx[at], *back["dx"], ref.U[typ])
        for name, g, b in zip(("dw_gate", "dw_up", "dw_down"), dw, before):
            near(f"{name} of {e}", g[e], *added(*back[name], b if b is None else b[e], grad), ref.U[typ])


@pytest.mark.parametrize("typ,T,D,V,grad,accumulate", [s[1:] for s in SHAPES if s[0] == "loss"])
def test_loss_paths(ops, typ, T, D, V, grad, accumulate):
    typ, grad = TYPES[typ], TYPES[grad]
    gen = torch.Generator(device="cuda").manual_seed(9)
    target = torch.randint(0, V, (T,), generator=gen, device="cuda")
    w = normal((V, D), typ, 1, 3 * D ** -0.5)
    x = (normal((T, D), torch.float32, 2) + w[target].float()).to(typ)
    target = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.1, -100, target)
    dloss = torch.rand(T, generator=gen, device="cuda").add_(0.5).div_(T)
    loss, lse = ops.cross_entropy_forward(x, w, target)
    dw, before = gradient((V, D), grad, accumulate, 3)
    if accumulate:
        before = before / T           # of the size of what is added
        dw.copy_(before)
    dx, _ = ops.cross_entropy_backward(dloss, x, w, target, lse, dw=dw, accumulate=bool(accumulate))
    want = exp.cross_entropy(x, w, target, -100, typ, dloss, grad)
    for name, got in (("loss", loss), ("lse", lse)):
        v, b = want[name]
        assert bool(((got.double() - v).abs() <= b).all()), name
    near("dx", dx, *want["dx"], ref.U[typ])
    near("dw", dw, *added(*want["dw"], before, grad), ref.U[typ])
