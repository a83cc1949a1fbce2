"""Measured jobs: gated feed-forward sub-layers run on the layer operators
(layer.py), timed on this GPU, as rows of the estimator's job tables.

The paper profiles a job's operators on a single GPU and prices plans from those
times (Sec. 3.4).  `FeedForwardLayer` is such a layer's training step: norm,
gated feed-forward block, norm with gate and residual, their gradients, and the
orthogonalised update of its weights.  `profile_layer` times it, `measured_job`
makes a job of such layers for `workloads.from_lists`, and the module's command
does all of it and prints the plans that the estimator finds:

    python -m paper_2403_16125_amd.layer_profile --model 1024 --layers 24 --batch 128
"""
from __future__ import annotations

import argparse
import dataclasses

from . import workloads
from .layer import LayerOps


class FeedForwardLayer:
    """r = x + scale * gate * norm(ffn(norm(x))), x a float32 stream, the block in
    `dtype`.  Weights are float32 masters with copies in `dtype` for the
    products; gradients come in `dtype`, momenta are float32."""

    def __init__(self, ops: LayerOps, model: int, inner: int, *, dtype=None, activation="silu", kind="rms",
                 scale=1.0, seed=0):
        torch = ops.torch
        self.ops, self.model, self.inner = ops, model, inner
        self.dtype = dtype or torch.bfloat16
        self.activation, self.norm = activation, dict(kind=kind)
        self.scale = scale
        gen = torch.Generator(device=ops.dev).manual_seed(seed)

        def normal(rows, cols):
            return torch.randn(rows, cols, generator=gen, device=ops.dev) * cols ** -0.5

        self.master = [normal(inner, model), normal(inner, model), normal(model, inner)]
        self.weights = [w.to(self.dtype) for w in self.master]
        self.momentum = [torch.zeros_like(w) for w in self.master]
        ones = lambda: torch.ones(model, dtype=self.dtype, device=ops.dev)
        self.w_pre, self.w_post, self.gate = ones(), ones(), ones()

    def forward(self, x):
        """(r, what backward reads) for the stream x [tokens, model]."""
        ops = self.ops
        _, n, s0 = ops.norm_forward(x, w_pre=self.w_pre, dtype=self.dtype, save=True, **self.norm)
        y, saved = ops.ffn_forward(n, *self.weights, activation=self.activation, save=True)
        r, _, s1 = ops.norm_forward(x, y, gate=self.gate, scale=self.scale, w_post=self.w_post, next_norm=False,
                                    save=True, **self.norm)
        return r, (x, n, s0, y, saved, r, s1)

    def backward(self, dr, kept):
        """(dx, gradients) from the gradient of r: those of the three weights, then
        of w_pre, w_post and gate."""
        ops = self.ops
        x, n, s0, y, saved, r, s1 = kept
        after = ops.norm_backward(None, dr, r, y, s1, gate=self.gate, scale=self.scale, w_post=self.w_post, **self.norm)
        dn, *dw = ops.ffn_backward(after["dy"], n, *self.weights, saved, activation=self.activation)
        before = ops.norm_backward(dn, after["dx"], x, None, s0, w_pre=self.w_pre, **self.norm)
        return before["dx"], [*dw, before["dw_pre"], after["dw_post"], after["dgate"]]

    def update(self, grads, rate: float, mu: float = 0.95) -> None:
        """Weights less rate times the orthogonal factor of their momentum, whose
        entries are of the size of 0.2 whatever the shape; the vectors less rate
        times their gradient."""
        for master, weight, momentum, g in zip(self.master, self.weights, self.momentum, grads):
            step = self.ops.orthogonal_update(g, momentum=momentum, mu=mu, dtype=self.dtype,
                                              scale=0.2 * max(g.shape) ** 0.5)
            master.add_(step, alpha=-rate)
            weight.copy_(master)
        for vector, g in zip((self.w_pre, self.w_post, self.gate), grads[3:]):
            vector.add_(g, alpha=-rate)

    def parameter_bytes(self) -> int:
        """Of the float32 masters, as the estimator's memory model counts them."""
        return 4 * (3 * self.model * self.inner + 3 * self.model)

    @staticmethod
    def kept_bytes(kept) -> int:
        """Of what a forward pass keeps for its backward pass, less the stream that
        the layer before keeps as its own r."""
        x, n, s0, y, saved, r, s1 = kept
        return sum(t.numel() * t.element_size() for t in (n, s0, y, saved.buffer, r, s1))


@dataclasses.dataclass
class LayerProfile:
    forward: float          # seconds
    backward: float
    update: float
    tokens: int             # of the measured pass
    parameter_bytes: int
    kept_bytes: int         # for the backward pass
    boundary_bytes: int     # the stream that the next layer reads


def profile_layer(layer: FeedForwardLayer, tokens: int, repeats: int = 5, passes: int = 4) -> LayerProfile:
    """Medians over `repeats` of `passes` passes each, after one to warm up."""
    torch = layer.ops.torch
    x = torch.randn(tokens, layer.model, device=layer.ops.dev)
    dr = torch.randn(tokens, layer.model, device=layer.ops.dev) / tokens

    def median(f):
        f()
        times = []
        for _ in range(repeats):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(passes):
                f()
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b) * 1e-3 / passes)
        return sorted(times)[repeats // 2]

    r, kept = layer.forward(x)
    _, grads = layer.backward(dr, kept)
    return LayerProfile(forward=median(lambda: layer.forward(x)), backward=median(lambda: layer.backward(dr, kept)),
                        update=median(lambda: layer.update(grads, 0.0)), tokens=tokens,
                        parameter_bytes=layer.parameter_bytes(), kept_bytes=layer.kept_bytes(kept),
                        boundary_bytes=r.numel() * r.element_size())


def measured_job(profiles, batch: int, seq: int = workloads.SEQ_LEN) -> dict:
    """A job for workloads.from_lists from its layers' profiles: times of the
    forward and backward pass scaled to a global batch of `batch` samples of
    `seq` tokens, bytes to one sample.  The speed-1 GPU is the one measured."""
    share = [seq / p.tokens for p in profiles]
    return dict(t=[(p.forward + p.backward) * s * batch for p, s in zip(profiles, share)],
                p=[p.parameter_bytes for p in profiles], a=[p.kept_bytes * s for p, s in zip(profiles, share)],
                x=[p.boundary_bytes * s for p, s in zip(profiles, share)], a2a=[0.0] * len(profiles), batch=batch)


# one MI355X node: 288 GB a GPU, a 153 GB/s xGMI link between each two of its 8 GPUs, a
# 400 Gbit/s network link a GPU
MI355X = dict(speed=1.0, mem=288e9, bw_intra=153e9, bw_inter=50e9, gpus_per_node=8)


def main(argv=None) -> None:
    from . import arena
    ap = argparse.ArgumentParser(description="Times a feed-forward layer on this GPU and estimates a job of such layers.")
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=0, help="default: 8/3 of --model, up to a multiple of 64")
    ap.add_argument("--layers", type=int, default=24)
    ap.add_argument("--batch", type=int, default=128, help="global batch, samples")
    ap.add_argument("--samples", type=int, default=4, help="samples of the measured pass")
    ap.add_argument("--seq", type=int, default=workloads.SEQ_LEN)
    a = ap.parse_args(argv)
    inner = a.inner or -(-a.model * 8 // 3 // 64) * 64
    ops = LayerOps()
    try:
        layer = FeedForwardLayer(ops, a.model, inner)
        p = profile_layer(layer, a.samples * a.seq)
    finally:
        ops.torch.cuda.synchronize()
        ops.close()
    print(f"layer {a.model} x {inner}, {p.tokens} tokens: forward {p.forward * 1e6:.1f} us, backward "
          f"{p.backward * 1e6:.1f} us, update {p.update * 1e6:.1f} us; parameters {p.parameter_bytes / 1e6:.1f} MB, kept "
          f"{p.kept_bytes / 1e6:.1f} MB, boundary {p.boundary_bytes / 1e6:.1f} MB", flush=True)
    w = workloads.from_lists([measured_job([p] * a.layers, a.batch, a.seq)], [MI355X], [1, 2, 4, 8, 16, 32],
                             [1, 2, 4, 8, 16])
    est = arena.Estimator(w)
    try:
        est.estimate()
        r = est.results()
    finally:
        est.close()
    for i, n in enumerate(w.counts):
        print(f"{n:3d} GPUs: {r['t_iter'][i] * 1e3:9.2f} ms an iteration, {r['thr'][i]:9.1f} samples/s, dp {r['dp'][i]} "
              f"tp {r['tp'][i]} pp {r['pp'][i]} m {r['m'][i]}", flush=True)


if __name__ == "__main__":
    main()
