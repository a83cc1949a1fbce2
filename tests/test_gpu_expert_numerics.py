"""The operators of a layer of experts and the loss where sizes or values are extreme:
activations far below zero, and tensors whose offsets pass 31 bits."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2403_16125_amd import layer
from test_gpu_experts import check_experts, check_moves, check_route, experts_inputs, plan_of
from test_gpu_layer import inside, normal
from test_gpu_loss import check as check_loss, inputs as loss_inputs

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
FAR = 1 << 20                 # row stride: 2100 rows of it pass 2^31 values


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()
    torch.cuda.empty_cache()


def far(t, stride=FAR):
    """t with its first axis `stride` values apart, NaN between."""
    mem = torch.full((t.shape[0], stride), math.nan if t.is_floating_point() else -1, dtype=t.dtype, device="cuda")
    v = mem[:, :t[0].numel()].unflatten(1, t.shape[1:])
    v.copy_(t)
    assert (t.shape[0] - 1) * stride >= 2 ** 31
    return v


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T", [1, 70, 1000])
@pytest.mark.parametrize("act,low", [("gelu", -8.0), ("gelu", -40.0), ("silu", -80.0)])
def test_activations_far_below_zero(ops, act, low, T, typ):
    """As of the feed-forward block (test_gpu_layer_numerics): one rounding of h (du, dg), and 2^-16 of
    the value for the arithmetic.  The exponent e of gelu's exponential carries e 2^-24 of rounding
    into it, at most 88 of them before it leaves the range; below that is the type's least step, and
    a result that is subnormal in 32 bits may be 0."""
    F = 128
    z = torch.linspace(low, 2.0, F, device="cuda").to(typ)
    x, wg, wu = torch.zeros(T, 8, dtype=typ, device="cuda"), *(torch.zeros(1, F, 8, dtype=typ, device="cuda") for _ in range(2))
    x[:, 0], wg[:, :, 0], wu[:, :, 0] = 1.0, z, 1024.0       # g = z, u = 1024
    wd = torch.zeros(1, 8, F, dtype=typ, device="cuda")
    offsets = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    _, saved = ops.experts_forward(x, offsets, wg, wu, wd, activation=act, save=True)
    h = saved.buffer[:2 * T * F].view(typ).view(T, F).double()
    g = z.double()
    if act == "gelu":
        c, p = torch.erfc(-g / 2 ** 0.5) / 2, torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
        value, slope, size = g * c, c + g * p, c + g.abs() * p
    else:
        s = 1 / (1 + torch.exp(-g))
        value, slope, size = g * s, s + g * s * (1 - s), s + g.abs() * s * (1 - s)
    least = ref.TINY[typ] + 1024 * 40 * 2.0 ** -126
    off = (h - 1024 * value).abs() - 1024 * value.abs() * (ref.U[typ] + 2.0 ** -16) - least
    assert off.max() <= 0, (g[off.amax(0).argmax()].item(), off.max().item())
    # dh = 1 for every feature: the gradients of the weights are T times du and dg
    wd[:, 0] = 1.0
    dy = torch.zeros(T, 8, dtype=typ, device="cuda")
    dy[:, 0] = 1.0
    grads = [torch.empty(w.shape, device="cuda") for w in (wg, wu, wd)]
    ops.experts_backward(dy, x, offsets, wg, wu, wd, saved, activation=act, grads=grads)
    du, dg = grads[1][0, :, 0].double() / T, grads[0][0, :, 0].double() / T
    much = 2.0 ** -16 + T * 2.0 ** -24                # and the sum over tokens
    off = (du - value).abs() - value.abs() * (ref.U[typ] + much) - least
    assert off.max() <= 0, (g[off.argmax()].item(), off.max().item())
    off = (dg - 1024 * slope).abs() - 1024 * (ref.U[typ] * slope.abs() + much * size) - least
    assert off.max() <= 0, (g[off.argmax()].item(), off.max().item())


def test_route_of_far_rows(ops):
    check_route(ops, far(normal((2100, 40), BF16, 1, 2.0)), 4, True)


def test_moves_of_far_rows(ops):
    T, D, k = 1100, 136, 2
    plan = plan_of(ops, T, k, 8, 3)
    ys, dxs = (far(normal((T * k, D), BF16, s)) for s in (2, 4))
    x, dy = normal((T, D), BF16, 1), normal((T, D), BF16, 3)
    outs = [far(torch.full((T * k, D), 7.0, dtype=BF16, device="cuda")) for _ in range(2)]
    check_moves(ops, x, ys, dy, dxs, plan, torch.rand(T, k, device="cuda"), [*outs, torch.full((T * k, D), 7.0, dtype=BF16, device="cuda"),
                                                                             None])


def test_moves_of_many_rows(ops):
    """600000 rows of 4096 values."""
    T, D, k = 300000, 4096, 2
    plan = plan_of_many(ops, T, k, 64)
    x = torch.empty(T, D, dtype=BF16, device="cuda").normal_()
    xs = ops.dispatch(x, plan)
    row = plan.row.long()
    for t in range(0, T, 50000):
        for j in range(k):
            assert torch.equal(xs[row[t:t + 50000, j]], x[t:t + 50000])
    # two equal rows halved each give the row again
    assert torch.equal(ops.combine(xs, plan, torch.full((T, k), 0.5, device="cuda")), x)
    weight = torch.full((T, k), 0.5, device="cuda")
    dys, dweight = ops.combine_backward(x, xs, plan, weight)
    at = torch.arange(T - 3000, T, device="cuda")
    assert torch.equal(dys[row[at, 1]], x[at] * 0.5)
    dots = (x[at].double() ** 2).sum(1)
    inside("dweight", dweight[at, 0], dots, dots * D * 2.0 ** -23)


def plan_of_many(ops, T, k, E):
    index = torch.rand(T, E, device="cuda").topk(k).indices
    return ops.sort_by_expert(index, E)


def test_experts_of_far_rows(ops):
    t = list(experts_inputs([900, 0, 1203], 72, 64, BF16))
    t[0], t[5] = far(t[0]), far(t[5])
    check_experts(ops, t, "silu", BF16)


@pytest.mark.parametrize("D", [72, 65])
@pytest.mark.parametrize("rows", [1, 30])
def test_experts_of_far_matrices(ops, rows, D):
    t = list(experts_inputs([rows] * 10, D, 136, F16))
    for i in (2, 3, 4):
        t[i] = far(t[i], 1 << 28)
    check_experts(ops, t, "gelu", F16)


def test_experts_gradients_of_far_matrices(ops):
    x, offsets, wg, wu, wd, dy = experts_inputs([30] * 10, 72, 136, BF16)
    _, saved = ops.experts_forward(x, offsets, wg, wu, wd, save=True)
    want = ops.experts_backward(dy, x, offsets, wg, wu, wd, saved)
    grads = [far(torch.zeros_like(w), 1 << 28) for w in (wg, wu, wd)]
    ops.experts_backward(dy, x, offsets, wg, wu, wd, saved, grads=grads, accumulate=False)
    for g, w in zip(grads, want[1:]):
        assert torch.equal(g, w)


@pytest.mark.parametrize("T,V", [(2100, 300), (9, 2200), (100, 2200)])
def test_loss_of_far_rows(ops, T, V):
    x, w, target, dloss = loss_inputs(T, 72, V, BF16)
    if T > 2000:
        x = far(x)
    else:
        w = far(w)
    check_loss(ops, x, w, target, dloss)


def test_loss_of_the_largest_vocabulary(ops):
    """2^24 entries of 8 values, few tokens: the logits' gradient has rows of 2^25 bytes."""
    T, D, V = 7, 8, 1 << 24
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, D, generator=gen, device="cuda").to(BF16)
    w = torch.randn(V, D, generator=gen, device="cuda").to(BF16)
    target = torch.tensor([0, V - 1, V // 2, 5, V - 2, -100, 77], device="cuda")
    check_loss(ops, x, w, target, torch.rand(T, generator=gen, device="cuda"))
