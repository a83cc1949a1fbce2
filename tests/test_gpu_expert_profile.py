"""Layers of experts and the loss as training steps, and as measured layers of the
estimator's jobs, on the GPU."""
import numpy as np
import pytest
import torch

import experts_reference as exp
import layer_reference as ref
from paper_2403_16125_amd import arena, layer_profile as lp, workloads
from paper_2403_16125_amd.layer import LayerOps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    o = LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def test_expert_layer_against_autograd(ops):
    """The whole layer, with the experts that its router chose, against differentiating the definition in
    64 bits: each gradient to 2 % of its norm, as the feed-forward layer's, but the router's,
    whose logits are formed from the rounded n of the layer: 2^-8 of each value of it at most, which the
    differences of weights that a gradient is made of take a few times larger, so 5 %."""
    E, k = 6, 2
    layer = lp.ExpertLayer(ops, 96, 160, E, k, scale=0.5, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dr = (torch.randn(70, 96, generator=gen, device="cuda") for _ in range(2))
    r, kept = layer.forward(x)
    index = kept[4][1].long()
    dx, grads = layer.backward(dr, kept)
    leaves = [t.double().requires_grad_() for t in (x, *layer.weights, layer.w_pre, layer.w_post, layer.gate, layer.router)]
    xd, wg, wu, wd, w_pre, w_post, gate, router = leaves
    n = ref.norm(xd, "rms", 1e-6)[0] * w_pre
    weight = exp.route_weight(n @ router.T, index, True, 1.0)
    y = 0
    for j in range(k):
        e = index[:, j]
        h = ref.act(torch.bmm(wg[e], n[:, :, None])[:, :, 0], "silu")[0] * torch.bmm(wu[e], n[:, :, None])[:, :, 0]
        y = y + weight[:, j:j + 1] * torch.bmm(wd[e], h[:, :, None])[:, :, 0]
    want = xd + 0.5 * gate * (ref.norm(y, "rms", 1e-6)[0] * w_post)
    assert (r.double() - want).norm() <= 0.02 * want.norm()
    for i, (got, g) in enumerate(zip((dx, *grads), torch.autograd.grad((want * dr.double()).sum(), leaves))):
        assert (got.double() - g).norm() <= (0.05 if i == 7 else 0.02) * g.norm(), i


def test_loss_layer_against_autograd(ops):
    layer = lp.LossLayer(ops, 64, 300, seed=5)
    (x, target), one = layer.sample(50)
    target[3:9] = layer.ignore_index
    loss, kept = layer.forward(x, target)
    dx, (dw,) = layer.backward(one, kept)
    xd, wd = (t.double().requires_grad_() for t in (x, layer.weight))
    want = torch.nn.functional.cross_entropy(xd @ wd.T, target, ignore_index=layer.ignore_index)
    assert abs(loss - want) <= 1e-4
    want.backward()
    # one rounding of the logits' gradient and one of the result, 2^-8 of a value each at most
    for got, g in ((dx, xd.grad), (dw, wd.grad)):
        assert (got.double() - g).norm() <= 2 * 2.0 ** -8 * g.norm()
    layer.update([dw], 0.5)
    assert torch.equal(layer.weight, layer.master.bfloat16())


def test_update_moves_every_parameter(ops):
    layer = lp.ExpertLayer(ops, 64, 80, 3, 1, seed=6)
    (x, dr) = layer.sample(40)
    before = [t.clone() for t in (*layer.master, layer.router)]
    _, kept = layer.forward(x)
    _, grads = layer.backward(dr, kept)
    layer.update(grads, 0.1)
    for b, t, g in zip(before, (*layer.master, layer.router), (*grads[:3], grads[6])):
        assert not g.any() or not torch.equal(b, t)
    assert torch.isfinite(layer.router).all()


def test_measured_layers_make_a_job(ops):
    kinds = [lp.FeedForwardLayer(ops, 256, 704), lp.ExpertLayer(ops, 256, 704, 4, 2), lp.LossLayer(ops, 256, 4096)]
    p = [lp.profile_layer(k, 1024, repeats=3, passes=2) for k in kinds]
    assert all(v.forward > 0 and v.backward > 0 and v.update > 0 for v in p)
    assert p[1].parameter_bytes == 4 * (4 * 3 * 256 * 704 + 3 * 256 + 4 * 256)
    assert p[1].all_to_all_bytes == 1024 * 2 * 256 * 2 and p[0].all_to_all_bytes == p[2].all_to_all_bytes == 0
    # n, y, xs, ys in 16 bits, r in 32, h in 16 and g, u in 24 bits, logits, indices, weights, rows, statistics
    assert abs(p[1].kept_bytes - 1024 * (8 * 256 + 2 * 4 * 256 + 2 * 8 * 704 + 4 * 4 + 3 * 8 + 32)) <= 2048
    assert p[2].parameter_bytes == 4 * 256 * 4096 and p[2].boundary_bytes == 4 and p[2].kept_bytes == 1024 * 12 + 4
    job = lp.measured_job([p[0], p[1], p[0], p[1], p[2]], 32)
    assert job["a2a"] == [0.0, p[1].all_to_all_bytes, 0.0, p[1].all_to_all_bytes, 0.0]
    w = workloads.from_lists([job], [lp.MI355X], [1, 2, 4, 8], [1, 2, 4])
    est = arena.Estimator(w)
    try:
        est.estimate()
        res = est.results()
    finally:
        est.close()
    assert (res["t_iter"] > 0).all() and np.isfinite(res["t_iter"]).all()


def test_command(capsys):
    lp.main(["--model", "256", "--layers", "4", "--batch", "16", "--samples", "1", "--experts", "4", "--vocabulary", "2000"])
    out = capsys.readouterr().out
    assert "4 experts" in out and "loss 256 x 2000" in out and " 32 GPUs:" in out
