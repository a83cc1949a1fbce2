"""The layer operators as a training step, and measured layers as jobs of the
estimator, on the GPU."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from compare import compare
from paper_2403_16125_amd import arena, layer_profile as lp, workloads
from paper_2403_16125_amd.layer import COEFFICIENTS, LayerOps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    o = LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def test_layer_against_autograd(ops):
    """Forward and backward of the whole layer against differentiating the definition in
    64 bits: each gradient to 2 % of its norm (six roundings of 2^-8 at most on
    the way, taken a few times larger by the norms)."""
    layer = lp.FeedForwardLayer(ops, 96, 160, scale=0.5, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dr = (torch.randn(70, 96, generator=gen, device="cuda") for _ in range(2))
    r, kept = layer.forward(x)
    dx, grads = layer.backward(dr, kept)
    leaves = [t.double().requires_grad_() for t in (x, *layer.weights, layer.w_pre, layer.w_post, layer.gate)]
    xd, wg, wu, wd, w_pre, w_post, gate = leaves
    n = ref.norm(xd, "rms", 1e-6)[0] * w_pre
    y = torch.mm(ref.act(torch.mm(n, wg.T), "silu")[0] * torch.mm(n, wu.T), wd.T)
    want = xd + 0.5 * gate * (ref.norm(y, "rms", 1e-6)[0] * w_post)
    assert (r.double() - want).norm() <= 0.02 * want.norm()
    for got, g in zip((dx, *grads), torch.autograd.grad((want * dr.double()).sum(), leaves)):
        assert (got.double() - g).norm() <= 0.02 * g.norm()


def test_training_lowers_the_loss(ops):
    """Forty steps on a fixed target."""
    layer = lp.FeedForwardLayer(ops, 64, 176, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(256, 64, generator=gen, device="cuda")
    target = x + torch.tanh(torch.mm(x, torch.randn(64, 64, generator=gen, device="cuda") * 0.2))
    losses = []
    for _ in range(40):
        r, kept = layer.forward(x)
        losses.append(float(((r - target) ** 2).mean()))
        _, grads = layer.backward(2 * (r - target) / r.numel(), kept)
        layer.update(grads, 0.02)
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0], (losses[0], losses[-1])


def test_update_is_the_operators(ops):
    layer = lp.FeedForwardLayer(ops, 48, 80, seed=7)
    grads = [torch.randn_like(w) for w in layer.weights] + [torch.zeros(48, dtype=torch.bfloat16, device="cuda")] * 3
    before = [w.clone() for w in layer.master]
    layer.update(grads, 0.1, mu=0.0)
    for w, b, g, half in zip(layer.master, before, grads, layer.weights):
        want = b.double() - 0.1 * ref.orthogonal(g, COEFFICIENTS, 5, 1e-7, 0.2 * max(g.shape) ** 0.5)
        assert (w.double() - want).norm() <= 1e-2 * (want - b.double()).norm()
        assert torch.equal(half, w.bfloat16())


def test_measured_jobs_are_estimated(ops, oracle):
    """Measured layers go through the estimator, cell by cell as the oracle prices them."""
    profiles = {}
    for model, inner in ((256, 704), (512, 1376)):
        p = profiles[model] = lp.profile_layer(lp.FeedForwardLayer(ops, model, inner), 1024, repeats=3, passes=2)
        assert p.forward > 0 and p.backward > 0 and p.update > 0
        assert p.parameter_bytes == 4 * (3 * model * inner + 3 * model)
        assert p.boundary_bytes == 1024 * model * 4
        # n and y in 16 bits, r in 32, h in 16 and g, u in 24 bits, two rows of 4 statistics
        assert abs(p.kept_bytes - 1024 * (8 * model + 8 * inner + 32)) <= 1024
    jobs = [lp.measured_job([profiles[256]] * 8, 32), lp.measured_job([profiles[512], profiles[256]] * 6, 64)]
    assert jobs[0]["t"][0] == pytest.approx((profiles[256].forward + profiles[256].backward) * 32)
    w = workloads.from_lists(jobs, [lp.MI355X, dict(lp.MI355X, speed=0.5, mem=96e9)], [1, 2, 4, 8, 16], [1, 2, 4, 8])
    est = arena.Estimator(w, with_cuts=True)
    try:
        est.estimate()
        res = est.results()
    finally:
        est.close()
    rep = compare(w, res, np.arange(w.n_cells), oracle)
    assert not rep["mismatch"] and rep["n"] == w.n_cells
    assert (res["t_iter"] > 0).all() and np.isfinite(res["t_iter"]).all()


def test_command(capsys):
    lp.main(["--model", "256", "--layers", "4", "--batch", "16", "--samples", "1"])
    out = capsys.readouterr().out
    assert "forward" in out and " 32 GPUs:" in out
