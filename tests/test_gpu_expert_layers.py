"""Training steps of a layer of experts on the GPU: what each parameter's gradient and
update are, with several choices a token and with one."""
import pytest
import torch

import experts_reference as exp
import layer_reference as ref
from paper_2403_16125_amd import layer_profile as lp
from paper_2403_16125_amd.layer import LayerOps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    o = LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def test_every_parameter_has_a_gradient_and_moves_along_it(ops):
    layer = lp.ExpertLayer(ops, 64, 80, 3, 2, seed=6)
    x, dr = layer.sample(40)
    vectors = (layer.w_pre, layer.w_post, layer.gate, layer.router)
    before, masters = [t.clone() for t in vectors], [t.clone() for t in layer.master]
    _, kept = layer.forward(x)
    _, grads = layer.backward(dr, kept)
    layer.update(grads, 0.1)
    assert len(grads) == 7
    for i, g in enumerate(grads):
        assert bool(g.any()) and bool(torch.isfinite(g).all()), i
    for b, t, g in zip(before, vectors, grads[3:]):
        want = b.double() - 0.1 * g.double()
        # in 32 bits the product and the sum are rounded, then the result to its type
        off = 2.0 ** -23 * (0.1 * g.double().abs() + b.double().abs()) + ref.U[t.dtype] * want.abs() + ref.TINY[t.dtype]
        assert bool(((t.double() - want).abs() <= off).all())
    for b, t in zip(masters, layer.master):
        assert not torch.equal(b, t) and bool(torch.isfinite(t).all())


def test_one_choice_has_no_gradient_for_its_router(ops):
    """Not for want of a weight: in 64 bits, with the softmax over all experts as the weight, the norm behind the
    block leaves of the router's gradient what its epsilon (1e-6 beside a mean square of 1e-3 and more) does not
    cancel, less than the rounding of dy to 16 bits."""
    layer = lp.ExpertLayer(ops, 96, 160, 6, 1, scale=0.5, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dr = (torch.randn(70, 96, generator=gen, device="cuda") for _ in range(2))
    r, kept = layer.forward(x)
    _, index, weight = kept[4][:3]
    assert bool((weight == 1).all())
    dx, grads = layer.backward(dr, kept)
    assert not grads[6].any() and all(bool(g.any()) for g in grads[:6])
    xd, *ws = [t.double() for t in (x, *layer.weights)]
    router = layer.router.double().requires_grad_()
    n = ref.norm(xd, "rms", 1e-6)[0]
    e = index[:, 0].long()
    h = ref.act(torch.bmm(ws[0][e], n[:, :, None])[:, :, 0], "silu")[0] * torch.bmm(ws[1][e], n[:, :, None])[:, :, 0]
    v = torch.bmm(ws[2][e], h[:, :, None])[:, :, 0]
    through = lambda y: torch.autograd.grad((y * dr.double()).sum(), router, retain_graph=True)[0].norm()
    y = exp.route_weight(n @ router.T, e[:, None], False, 1.0) * v
    assert bool((y ** 2).mean(1).min() > 1e-3)
    assert through(ref.norm(y, "rms", 1e-6)[0]) <= 2.0 ** -8 * through(y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_routers_share_of_dn_is_added_in_32_bits(ops, dtype):
    """dn is the experts' share (a tensor of 16 bits) and the router's in one rounding of their sum: u of it, and what 32
    bits leave of the router's product of 6 and of the sum."""
    layer = lp.ExpertLayer(ops, 96, 160, 6, 2, dtype=dtype, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    n, dy = (torch.randn(200, 96, generator=gen, device="cuda").to(dtype) for _ in range(2))
    layer.router.mul_(4)        # of the experts' share's size
    _, kept = layer.block(n)
    dn, _, _ = layer.block_backward(dy, n, kept)
    logits, index, weight, plan, xs, ys, inner = kept
    dys, dweight = ops.combine_backward(dy, ys, plan, weight)
    dxs, *_ = ops.experts_backward(dys, xs, plan.offsets, *layer.weights, inner)
    own = ops.dispatch_backward(dxs, plan).double()
    dlogits = ops.route_backward(dweight, logits, index).double()
    share, size = dlogits @ layer.router.double(), dlogits.abs() @ layer.router.double().abs()
    want = own + share
    off = (dn.double() - want).abs()
    assert bool((off <= ref.U[dtype] * want.abs() + 8 * 2.0 ** -23 * (size + own.abs()) + ref.TINY[dtype]).all())
    assert bool((share.abs() > 2.0 ** -4 * own.abs()).float().mean() > 0.5)
