"""The cross entropy's gradients of up to 32 tokens, whose logits' gradient is kept in two
operands: off by what 32 bits leave of logits and probabilities and by one rounding of the
result, not by the rounding of a token's largest entry."""
import math

import pytest
import torch

import experts_reference as exp
from layer_reference import TINY, U
from paper_2403_16125_amd import layer
from test_gpu_layer import inside, normal, strided

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def inputs(T, D, V, typ, seed=1):
    """As of a model that has learnt: x leans towards its target's row."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.randint(0, V, (T,), generator=gen, device="cuda")
    w = normal((V, D), typ, seed, 3 * D ** -0.5)
    x = (normal((T, D), F32, seed + 1) + w[target].float()).to(typ)
    return x, w, target, torch.rand(T, generator=gen, device="cuda") + 0.5


def gradients(x, w, target, dloss, typ, grad_typ, ignore=-100):
    """{name: (value, bound)}: as experts_reference.cross_entropy's, but for the rounding of the logits'
    gradient g, u^2 of it here (and in float16 the least subnormal, with the largest dloss at 2^10 or more)."""
    x, w = x.double(), w.double()
    counted = target != ignore
    at = torch.where(counted, target, 0)[:, None]
    D, T, V = x.shape[1], x.shape[0], w.shape[0]
    l, bl = x @ w.T, D * 2.0 ** -23 * (x.abs() @ w.abs().T)
    lse = torch.logsumexp(l, 1)
    off = bl + (bl.amax(1) + 2.0 ** -15 + 2.0 ** -22 * lse.abs())[:, None] + 2.0 ** -15
    x = torch.where(counted[:, None], x, 0.0)
    dl = torch.where(counted, dloss.double(), 0.0)[:, None]
    p = torch.exp(l - lse[:, None])
    g = p.scatter_add(1, at, torch.full_like(dl, -1.0)) * dl
    least = TINY[typ] * (float(dl.abs().max()) * 2.0 ** -10 if typ is F16 else 1.0)
    bg = dl.abs() * (p * off * torch.exp(off) + 2.0 ** -23) + U[typ] ** 2 * g.abs() + least
    bg = torch.where(counted[:, None], bg, 0.0)
    out = {}
    for name, v, b, t in (("dx", g @ w, (bg + 2 * V * 2.0 ** -23 * g.abs()) @ w.abs(), typ),
                          ("dw", g.T @ x, (bg + 2 * T * 2.0 ** -23 * g.abs()).T @ x.abs(), grad_typ)):
        out[name] = v, b * (1 + U[t]) + U[t] * v.abs() + TINY[t]
    return out


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T,D,V", [(1, 64, 257), (1, 1, 1), (2, 130, 63), (7, 9, 5), (16, 65, 640), (31, 200, 1000), (32, 72, 513),
                                   (32, 512, 4001), (5, 1024, 30000)])
def test_gradients_of_few_tokens(ops, T, D, V, typ):
    x, w, target, dloss = inputs(T, D, V, typ)
    if T > 4:
        target[1] = target[2]           # one entry twice, and a token that does not count
        target[3] = -100
    _, lse = ops.cross_entropy_forward(x, w, target)
    for grad in (F32, typ):
        dw = torch.empty(V, D, dtype=grad, device="cuda")
        dx, _ = ops.cross_entropy_backward(dloss, x, w, target, lse, dw=dw)
        want = gradients(x, w, target, dloss, typ, grad)
        inside("dx", dx, *want["dx"])
        inside("dw", dw, *want["dw"])
    only, _ = ops.cross_entropy_backward(dloss, strided(x, 3, 1), strided(w, 3, 1), target, lse)
    inside("dx of uneven rows", only, *want["dx"])


@pytest.mark.parametrize("typ", [BF16, F16])
def test_few_tokens_in_pieces_and_added(ops, typ):
    """More than one piece of the vocabulary: 2 x 20 rows of 3.5 million entries; dw is added to."""
    T, D, V = 20, 4, 3500000
    x, w, target, dloss = inputs(T, D, V, typ)
    target[:3] = torch.tensor([0, V - 1, V // 2])
    _, lse = ops.cross_entropy_forward(x, w, target)
    dw = torch.full((V, D), 0.25, device="cuda")
    dx, _ = ops.cross_entropy_backward(dloss, x, w, target, lse, dw=dw, accumulate=True)
    want = gradients(x, w, target, dloss, typ, F32)
    inside("dx", dx, *want["dx"])
    v, b = want["dw"]
    inside("dw", dw, v + 0.25, b + U[F32] * (v + 0.25).abs())


def test_few_tokens_that_do_not_count(ops):
    """NaN in a token that the loss leaves out reaches nothing, in neither operand's rows; infinite gradients stay."""
    x, w, target, dloss = inputs(9, 64, 300, BF16)
    target[4] = -100
    _, lse = ops.cross_entropy_forward(x, w, target)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse)
    bad, d = x.clone(), dloss.clone()
    bad[4], d[4] = math.nan, math.inf
    _, lse2 = ops.cross_entropy_forward(bad, w, target)
    dx2, dw2 = ops.cross_entropy_backward(d, bad, w, target, lse2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and not dx[4].any()
    # past the largest bfloat16 an entry is infinite, and so are its products, not NaN
    d[:] = 0.0
    d[0] = 3.4e38
    w1, x1 = torch.ones_like(w), torch.ones_like(x)
    w1[int(target[0])] = 2.0
    _, lse3 = ops.cross_entropy_forward(x1 * 0, w1, target)
    dw3 = torch.empty(300, 64, device="cuda")
    ops.cross_entropy_backward(d, x1, w1, target, lse3 + 100.0, dw=dw3)
    # logits 64 and, the target's, 128; lse log 300 + 100: the entry is 3.4e38 (e^22 - 1)
    assert bool((dw3[int(target[0])] == math.inf).all())
    ops.cross_entropy_backward(d, x1, w1 * 0, target, lse3 + 100.0, dw=dw3)
    # logits 0: the entry is -3.4e38, which bfloat16 rounds to -inf
    assert bool((dw3[int(target[0])] == -math.inf).all())


def test_few_tokens_captured_and_replayed(ops):
    static = list(inputs(12, 96, 1000, F16))

    def run():
        loss, lse = ops.cross_entropy_forward(*static[:3])
        return [loss, *ops.cross_entropy_backward(static[3], *static[:3], lse)]

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for seed in (5, 6, 7):
        for s, n in zip(static, inputs(12, 96, 1000, F16, seed)):
            s.copy_(n)
        want = run()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
