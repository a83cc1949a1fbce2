"""The cross entropy of tokens whose target has nearly all of the probability: a loss of
1e-7 to 1e-4 is held to what 32 bits leave of a sum of about 1, not of its logarithm of 30 to 120.

Logits are whole numbers, so they are exact.  Of the 4 entries the target's exponential is 1 and the others'
exp(-gap); the sum adds up at most 3 of a lane's columns, 2 shuffles, 4 waves and 10 levels of the join
to it, each off by 2^-24 of a sum of about 1 where it adds something at all: with 3 entries beside the
target no more than 3 additions do.  An exponential is off by (gap + 4) 2^-24 of itself, the logarithm by 2^-22 of
itself."""
import math

import pytest
import torch

import experts_reference as exp
from paper_2403_16125_amd import layer

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
GAPS = (9, 10, 11, 12, 13, 14, 15, 16)


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def inputs(top, D, T, typ):
    """Token t's target is t % 4, its logit `top`, the others' `top` less a gap."""
    w = torch.zeros(4, D, device="cuda")
    w[:, 0] = 1.0
    w[range(4), range(1, 5)] = 1.0
    target = torch.arange(T, device="cuda") % 4
    gap = torch.tensor(GAPS, device="cuda")[torch.arange(T, device="cuda") // 4 % len(GAPS)]
    x = torch.zeros(T, D, device="cuda")
    x[:, 0] = (top - gap).float()
    x[torch.arange(T, device="cuda"), 1 + target] = gap.float()
    return x.to(typ), w.to(typ), target, gap.double()


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T", [1, 16, 40, 700, 5000])
@pytest.mark.parametrize("top,D", [(30, 8), (120, 8), (30, 9), (120, 72)])
def test_loss_of_confident_tokens(ops, top, D, T, typ):
    x, w, target, gap = inputs(top, D, T, typ)
    loss, lse = ops.cross_entropy_forward(x, w, target)
    rest = 3 * torch.exp(-gap)
    want = torch.log1p(rest)
    off = (loss.double() - want).abs()
    assert bool((off <= 3 * 2.0 ** -24 * (1 + rest) + (gap + 4) * 2.0 ** -24 * rest + 2.0 ** -22 * want).all()), off.max()
    assert bool(((lse.double() - top - want).abs() <= 2.0 ** -24 * (top + 1) + 4 * 2.0 ** -24).all())
    # the difference from lse, rounded near `top`, would not do
    far = (lse.double() - top - want).abs()
    assert T < 16 or bool((far > 3 * 2.0 ** -24 * (1 + rest) + (gap + 4) * 2.0 ** -24 * rest + 2.0 ** -22 * want).any())


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T", [1, 40, 700])
@pytest.mark.parametrize("top", [30, 120])
def test_gradient_of_confident_tokens(ops, top, T, typ):
    """The target's entry of a row of the logits' gradient is off by lse's rounding, 2^-24 |lse| of dloss, and (an
    exponential near 1, the subtraction) 2^-22; another's by as much of its p, and by (gap + 4) 2^-24 of it: 16 times
    the target's is more than both.  Then it is rounded to 16 bits.  With one token that counts dw is that row times x."""
    x, w, target, gap = inputs(top, 8, T, typ)
    _, lse = ops.cross_entropy_forward(x, w, target)
    each = range(0, T, max(1, T // 8))
    for t in each:
        dloss = torch.zeros(T, device="cuda")
        dloss[t] = 1.0
        dw = torch.empty(4, 8, device="cuda")
        ops.cross_entropy_backward(dloss, x, w, target, lse, dw=dw)
        p = math.exp(-float(gap[t])) / (1 + 3 * math.exp(-float(gap[t])))
        u = exp.U[typ]
        least = 2.0 ** -24 * 2.0 ** -10 if typ is F16 else 0.0
        for v in range(4):
            mine = v == int(target[t])
            g = -3 * p if mine else p
            off = (2.0 ** -24 * (top + 1) + 2.0 ** -22) * (1.0 if mine else p * 16) + u * abs(g) + least
            assert bool(((dw[v].double() - g * x[t].double()).abs() <= (off + 2.0 ** -23 * abs(g)) * x[t].double().abs()).all()), (t, v)
