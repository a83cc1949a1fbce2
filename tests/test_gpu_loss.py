"""The cross entropy over a vocabulary on the GPU against its definition in 64 bits, by
the elementwise bounds of experts_reference."""
import math

import pytest
import torch

import experts_reference as exp
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


def inputs(T, D, V, typ, ignored=0.2, ignore=-100, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.randint(0, V, (T,), generator=gen, device="cuda")
    w = normal((V, D), typ, seed, 3 * D ** -0.5)
    x = (normal((T, D), F32, seed + 1) + w[target].float()).to(typ)
    target = torch.where(torch.rand(T, generator=gen, device="cuda") < ignored, ignore, target)
    return x, w, target, torch.rand(T, generator=gen, device="cuda").add_(0.5).div_(T)


def check(ops, x, w, target, dloss, ignore=-100, grad_typ=None, **given):
    typ = x.dtype
    loss, lse = ops.cross_entropy_forward(x, w, target, ignore_index=ignore)
    want = exp.cross_entropy(x, w, target, ignore, typ, dloss, grad_typ)
    inside("loss", loss, *want["loss"])
    inside("lse", lse, *want["lse"])
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse, ignore_index=ignore, **given)
    inside("dx", dx, *want["dx"])
    inside("dw", dw, *want["dw"])
    return loss, lse, dx, dw


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T,D,V", [(1, 1, 1), (1, 64, 257), (2, 8, 2), (3, 130, 63), (16, 65, 64), (33, 72, 65), (64, 128, 1000),
                                   (65, 200, 513), (130, 64, 4097), (257, 96, 300), (1024, 40, 777), (1100, 24, 129)])
def test_loss(ops, T, D, V, typ):
    check(ops, *inputs(T, D, V, typ))


@pytest.mark.parametrize("T,D,V,typ", [(777, 1000, 5001, F16), (1024, 512, 32768, BF16), (2048, 1024, 4096, BF16), (1, 4096, 20000, BF16),
                                       (300, 2048, 10000, F16)])
def test_loss_larger(ops, T, D, V, typ):
    check(ops, *inputs(T, D, V, typ))


@pytest.mark.parametrize("typ", [BF16, F16])
def test_loss_in_pieces_of_the_vocabulary(ops, typ):
    """More than one piece: 4096 x 40000 values of the logits' gradient pass what a call holds."""
    check(ops, *inputs(4096, 72, 40000, typ))


def test_loss_in_pieces_of_the_tokens(ops):
    x, w, target, dloss = inputs(33000, 16, 300, BF16)
    check(ops, x, w, target, dloss)


@pytest.mark.parametrize("ignore", [-100, 0, 7, -1])
def test_ignored_tokens_count_for_nothing(ops, ignore):
    """Whatever their rows, gradients and sums hold; an index of the vocabulary can be the ignored one."""
    x, w, target, dloss = inputs(100, 72, 50, BF16, 0.4, ignore)
    off = target == ignore
    loss, lse, dx, dw = check(ops, x, w, target, dloss, ignore)
    bad = x.clone()
    bad[off] = math.nan
    bad[off.nonzero()[0]] = math.inf
    d = dloss.clone()
    d[off] = math.inf
    loss2, lse2 = ops.cross_entropy_forward(bad, w, target, ignore_index=ignore)
    dx2, dw2 = ops.cross_entropy_backward(d, bad, w, target, lse2, ignore_index=ignore)
    assert torch.equal(loss, loss2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    assert torch.equal(lse[~off], lse2[~off]) and not loss[off].any() and not dx[off].any()


@pytest.mark.parametrize("typ", [BF16, F16])
def test_all_tokens_ignored(ops, typ):
    x, w, target, dloss = inputs(70, 64, 100, typ, 2.0)
    loss, lse = ops.cross_entropy_forward(x, w, target)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse)
    assert not loss.any() and not dx.any() and not dw.any()


def test_targets_outside_of_the_vocabulary(ops):
    x, w, target, dloss = inputs(20, 64, 100, BF16, 0.0)
    target[3], target[5] = 100, -7
    loss, lse = ops.cross_entropy_forward(x, w, target)
    assert torch.isnan(loss).nonzero().flatten().tolist() == [3, 5] and not torch.isnan(lse).any()
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse)
    assert torch.isnan(dx).any(1).nonzero().flatten().tolist() == [3, 5] and torch.isnan(dw).all()


def test_logits_that_are_not_finite(ops):
    x, w, target, _ = inputs(6, 64, 100, BF16, 0.0)
    target[:] = 50
    w[10] = 0.0
    x[1, 3] = math.nan
    x[2, 5], w[20] = math.inf, 0.0
    w[20, 5] = 1.0
    loss, lse = ops.cross_entropy_forward(x, w, target)
    assert torch.isnan(loss[1]) and torch.isnan(loss[2])
    assert torch.isfinite(loss[[0, 3, 4, 5]]).all()
    # a masked entry of the vocabulary: -inf logits have no share
    x = x.nan_to_num(0.0, 0.0).abs()
    w[10, 0] = -math.inf
    x[:, 0] = 1.0
    loss, lse = ops.cross_entropy_forward(x, w, target)
    keep = torch.arange(100, device="cuda") != 10
    want = torch.logsumexp(x.double() @ w.double()[keep].T, 1)
    assert (lse.double() - want).abs().max() < 1e-4        # bound: 64 products of up to 20, 2^-23 each, and 2^-15


def test_large_logits(ops):
    """Logits of some thousands, and all alike."""
    x, w, target, dloss = inputs(40, 64, 300, BF16, 0.0)
    check(ops, x * 30, w, target, dloss)
    loss, lse = ops.cross_entropy_forward(x * 0, w, target)
    assert (lse - math.log(300)).abs().max() < 2.0 ** -14


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("pad,offset", [(0, 1), (8, 0), (3, 0), (24, 8), (1, 5)])
def test_strides_and_alignment(ops, T, pad, offset):
    x, w, target, dloss = inputs(T, 96, 333, BF16)
    check(ops, strided(x, pad, offset), strided(w, pad, offset), target, dloss)


@pytest.mark.parametrize("typ", [BF16, F16])
def test_target_and_gradient_forms(ops, typ):
    x, w, target, _ = inputs(60, 72, 333, typ)
    loss, lse, dx, dw = check(ops, x, w, target, torch.full((60,), 0.125, device="cuda"))
    for d in (torch.tensor(0.125, device="cuda"), torch.tensor(0.125, device="cuda").expand(60),
              torch.full((60, 3), 0.125, device="cuda")[:, 1]):
        got = ops.cross_entropy_backward(d, x, w, target.int(), lse)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    a, b = ops.cross_entropy_forward(x.view(6, 10, 72), w, target.int().view(6, 10))
    assert torch.equal(a.view(-1), loss) and torch.equal(b.view(-1), lse)
    dx3, _ = ops.cross_entropy_backward(torch.tensor(0.125, device="cuda"), x.view(6, 10, 72), w, target.view(6, 10), b)
    assert torch.equal(dx3.view(60, 72), dx)


@pytest.mark.parametrize("much", [1e-30, 1e-6, 1.0, 65536.0, 1e30])
def test_float16_takes_gradients_of_any_size(ops, much):
    """A power of two brings them into float16's range and back; results past it overflow as any conversion."""
    x, w, target, dloss = inputs(100, 64, 400, F16)
    _, lse = ops.cross_entropy_forward(x, w, target)
    dw = torch.empty(w.shape, device="cuda")
    d = dloss * much
    ops.cross_entropy_backward(d, x, w, target, lse, dw=dw)
    want = exp.cross_entropy(x, w, target, -100, F16, d, F32)["dw"]
    inside("dw", dw, *want)


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T,D,V", [(130, 200, 328), (2000, 64, 100)])
def test_float_gradient_accumulates(ops, T, D, V, typ):
    x, w, target, dloss = inputs(T, D, V, typ)
    _, lse, _, low = check(ops, x, w, target, dloss)
    first = torch.empty(w.shape, device="cuda")
    ops.cross_entropy_backward(dloss, x, w, target, lse, dw=first)
    assert torch.equal(first.to(typ), low)
    box = torch.full((V + 2, D + 7), 0.5, device="cuda")
    view = box[1:-1, 3:-4]
    ops.cross_entropy_backward(dloss, x, w, target, lse, dw=view, accumulate=True)
    v, bound = exp.cross_entropy(x, w, target, -100, typ, dloss, F32)["dw"]
    inside("+ 0.5", view, v + 0.5, bound + (v + 0.5).abs() * 2.0 ** -24)
    view.fill_(0.5)
    assert bool((box == 0.5).all())


@pytest.mark.parametrize("typ", [BF16, F16])
def test_no_tokens(ops, typ):
    x, w, target, dloss = inputs(0, 64, 100, typ)
    loss, lse = ops.cross_entropy_forward(x, w, target)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse)
    assert loss.shape == lse.shape == (0,) and dx.shape == (0, 64) and not dw.any()
    kept = torch.ones_like(w)
    ops.cross_entropy_backward(dloss, x, w, target, lse, dw=kept, accumulate=True)
    assert bool((kept == 1).all())


def test_against_differences(ops):
    """The gradient's step along itself changes the mean loss, from 64 bits of the formula, as it says:
    second order is below the step."""
    x, w, target, _ = inputs(50, 64, 200, BF16, 0.1)
    loss, lse = ops.cross_entropy_forward(x, w, target)
    dx, dw = ops.cross_entropy_backward(torch.tensor(1.0, device="cuda"), x, w, target, lse)
    at = lambda s: exp.cross_entropy(x.double() + s * dx.double(), w.double() + s * dw.double(), target, -100, BF16)["loss"][0].sum()
    h = 1e-5
    slope = (at(h) - at(-h)) / (2 * h)
    size = dx.double().norm() ** 2 + dw.double().norm() ** 2
    assert abs(slope - size) <= 2 * 2.0 ** -8 * size


def test_captured_and_replayed(ops):
    static = list(inputs(200, 96, 1000, F16))

    def run():
        loss, lse = ops.cross_entropy_forward(*static[:3])
        return [loss, *ops.cross_entropy_backward(static[3], *static[:3], lse)]

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for seed in (5, 6, 7):
        for s, n in zip(static, inputs(200, 96, 1000, F16, seed=seed)):
            s.copy_(n)
        want = run()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_on_another_stream(ops):
    x, w, target, dloss = inputs(200, 96, 1000, BF16)
    _, lse, dx, dw = check(ops, x, w, target, dloss)
    s = torch.cuda.Stream()
    loss2, lse2 = ops.cross_entropy_forward(x, w, target, stream=s)
    dx2, dw2 = ops.cross_entropy_backward(dloss, x, w, target, lse2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(lse, lse2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
