"""Measured jobs: layers run on the layer operators (layer.py), timed on this GPU,
as rows of the estimator's job tables.

The paper profiles a job's operators on a single GPU and prices plans from those
times (Sec. 3.4).  `FeedForwardLayer` is such a layer's training step: norm,
gated feed-forward block, norm with gate and residual, their gradients, and the
orthogonalised update of its weights.  `ExpertLayer` has a mixture of experts in
the block's place, as every other layer of the MoE jobs; `LossLayer` is what ends a
language model's stack, the cross entropy over its vocabulary.  `profile_layer` times
them, `measured_job` makes a job of such layers for `workloads.from_lists`, and the
module's command does all of it and prints the plans that the estimator finds:

    python -m paper_2403_16125_amd.layer_profile --model 1024 --layers 24 --batch 128
    python -m paper_2403_16125_amd.layer_profile --experts 8 --choices 2 --vocabulary 32768
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

    stack = ()              # axes before those of a weight

    def __init__(self, ops: LayerOps, model: int, inner: int, *, dtype=None, activation="silu", kind="rms",
                 scale=1.0, seed=0):
        torch = ops.torch
        self.ops, self.model, self.inner = ops, model, inner
        self.dtype = dtype or torch.bfloat16
        self.activation, self.norm = activation, dict(kind=kind)
        self.scale = scale
        self.gen = gen = torch.Generator(device=ops.dev).manual_seed(seed)

        def normal(rows, cols):
            return torch.randn(*self.stack, rows, cols, generator=gen, device=ops.dev) * cols ** -0.5

        self.master = [normal(inner, model), normal(inner, model), normal(model, inner)]
        self.weights = [w.to(self.dtype) for w in self.master]
        self.momentum = [torch.zeros_like(w) for w in self.master]
        ones = lambda: torch.ones(model, dtype=self.dtype, device=ops.dev)
        self.w_pre, self.w_post, self.gate = ones(), ones(), ones()

    def forward(self, x):
        """(r, what backward reads) for the stream x [tokens, model]."""
        ops = self.ops
        _, n, s0 = ops.norm_forward(x, w_pre=self.w_pre, dtype=self.dtype, save=True, **self.norm)
        y, saved = self.block(n)
        r, _, s1 = ops.norm_forward(x, y, gate=self.gate, scale=self.scale, w_post=self.w_post, next_norm=False,
                                    save=True, **self.norm)
        return r, (x, n, s0, y, saved, r, s1)

    def block(self, n):
        """(y, what its backward pass reads)."""
        return self.ops.ffn_forward(n, *self.weights, activation=self.activation, save=True)

    def block_backward(self, dy, n, saved):
        """(dn, gradients of the three weights, those of other parameters)."""
        dn, *dw = self.ops.ffn_backward(dy, n, *self.weights, saved, activation=self.activation)
        return dn, dw, []

    def backward(self, dr, kept):
        """(dx, gradients) from the gradient of r: those of the three weights, then
        of w_pre, w_post and gate, then of what the block has more."""
        ops = self.ops
        x, n, s0, y, saved, r, s1 = kept
        after = ops.norm_backward(None, dr, r, y, s1, gate=self.gate, scale=self.scale, w_post=self.w_post, **self.norm)
        dn, dw, more = self.block_backward(after["dy"], n, saved)
        before = ops.norm_backward(dn, after["dx"], x, None, s0, w_pre=self.w_pre, **self.norm)
        return before["dx"], [*dw, before["dw_pre"], after["dw_post"], after["dgate"], *more]

    def update(self, grads, rate: float, mu: float = 0.95) -> None:
        """Weights less rate times the orthogonal factor of their momentum, whose
        entries are of the size of 0.2 whatever the shape; the vectors less rate
        times their gradient."""
        for master, weight, momentum, g in zip(self.master, self.weights, self.momentum, grads):
            step = self.ops.orthogonal_update(g, momentum=momentum, mu=mu, dtype=self.dtype,
                                              scale=0.2 * max(g.shape[-2:]) ** 0.5)
            master.add_(step, alpha=-rate)
            weight.copy_(master)
        for vector, g in zip((self.w_pre, self.w_post, self.gate, *self.others()), grads[3:]):
            vector.add_(g, alpha=-rate)

    def others(self):
        """Parameters that the block has beside its three weights."""
        return ()

    def sample(self, tokens):
        """An input and a gradient of the output to measure with."""
        torch, dev = self.ops.torch, self.ops.dev
        return torch.randn(tokens, self.model, device=dev), torch.randn(tokens, self.model, device=dev) / tokens

    def all_to_all_bytes(self, tokens) -> int:
        """That `tokens` tokens send to other GPUs' experts and get back, each way."""
        return 0

    def parameter_bytes(self) -> int:
        """Of the float32 masters, as the estimator's memory model counts them."""
        return 4 * (sum(w.numel() for w in (*self.master, *self.others())) + 3 * self.model)

    @staticmethod
    def kept_bytes(kept) -> int:
        """Of what a forward pass keeps for its backward pass, less the stream that
        the layer before keeps as its own r."""
        x, n, s0, y, saved, r, s1 = kept
        return sum(t.numel() * t.element_size() for t in (n, s0, y, saved.buffer, r, s1))


class ExpertLayer(FeedForwardLayer):
    """The same with a mixture of `experts` gated blocks: each token goes through the
    `choices` experts whose logits n router^T are largest, their outputs weighted by
    the softmax over these.  With one choice the router has a gradient of zero: its weight
    is 1, and any other would be taken out again by the norm behind the block, so that only the
    experts learn."""

    def __init__(self, ops: LayerOps, model: int, inner: int, experts: int, choices: int, **given):
        self.experts, self.choices, self.stack = experts, choices, (experts,)
        super().__init__(ops, model, inner, **given)
        torch = ops.torch
        self.router = torch.randn(experts, model, generator=self.gen, device=ops.dev) * model ** -0.5

    def others(self):
        return (self.router,)

    def block(self, n):
        ops = self.ops
        logits = n.float() @ self.router.t()
        index, weight = ops.route(logits, self.choices)
        plan = ops.sort_by_expert(index, self.experts)
        xs = ops.dispatch(n, plan)
        ys, saved = ops.experts_forward(xs, plan.offsets, *self.weights, activation=self.activation, save=True)
        return ops.combine(ys, plan, weight), (logits, index, weight, plan, xs, ys, saved)

    def block_backward(self, dy, n, saved):
        ops = self.ops
        logits, index, weight, plan, xs, ys, inner = saved
        dys, dweight = ops.combine_backward(dy, ys, plan, weight)
        dxs, *dw = ops.experts_backward(dys, xs, plan.offsets, *self.weights, inner, activation=self.activation)
        dlogits = ops.route_backward(dweight, logits, index)
        # the sum of both is formed in 32 bits
        dn = (ops.dispatch_backward(dxs, plan) + dlogits @ self.router).to(n.dtype)
        return dn, dw, [dlogits.t() @ n.float()]

    def all_to_all_bytes(self, tokens) -> int:
        return tokens * self.choices * self.model * self.w_pre.element_size()

    @staticmethod
    def kept_bytes(kept) -> int:
        x, n, s0, y, (logits, index, weight, plan, xs, ys, inner), r, s1 = kept
        return sum(t.numel() * t.element_size() for t in (n, s0, y, logits, index, weight, plan.offsets, plan.row, xs, ys,
                                                          inner.buffer, r, s1))


class LossLayer:
    """The mean cross entropy of x w^T against a target token each: x in `dtype`, w
    [vocabulary, model] a float32 master with a copy in `dtype`.  Tokens whose target is
    ignore_index count for nothing."""

    def __init__(self, ops: LayerOps, model: int, vocabulary: int, *, dtype=None, ignore_index=-100, seed=0):
        torch = ops.torch
        self.ops, self.model, self.vocabulary, self.ignore_index = ops, model, vocabulary, ignore_index
        gen = torch.Generator(device=ops.dev).manual_seed(seed)
        self.master = torch.randn(vocabulary, model, generator=gen, device=ops.dev) * model ** -0.5
        self.weight = self.master.to(dtype or torch.bfloat16)

    def forward(self, x, target):
        """(mean loss over the counted tokens, what backward reads)."""
        loss, lse = self.ops.cross_entropy_forward(x, self.weight, target, ignore_index=self.ignore_index)
        share = 1.0 / (target != self.ignore_index).sum().clamp(min=1).float()
        return loss.sum() * share, (x, target, lse, share)

    def backward(self, dloss, kept):
        """(dx, [dw]) from the gradient of the mean."""
        x, target, lse, share = kept
        dx, dw = self.ops.cross_entropy_backward(dloss * share, x, self.weight, target, lse,
                                                 ignore_index=self.ignore_index)
        return dx, [dw]

    def update(self, grads, rate: float) -> None:
        self.master.add_(grads[0], alpha=-rate)
        self.weight.copy_(self.master)

    def sample(self, tokens):
        torch, dev = self.ops.torch, self.ops.dev
        x = torch.randn(tokens, self.model, device=dev).to(self.weight.dtype)
        return (x, torch.randint(0, self.vocabulary, (tokens,), device=dev)), torch.ones((), device=dev)

    def all_to_all_bytes(self, tokens) -> int:
        return 0

    def parameter_bytes(self) -> int:
        return 4 * self.master.numel()

    @staticmethod
    def kept_bytes(kept) -> int:
        """Of what a forward pass keeps, less x, which the layer before wrote."""
        return sum(t.numel() * t.element_size() for t in kept[1:])


@dataclasses.dataclass
class LayerProfile:
    forward: float          # seconds
    backward: float
    update: float
    tokens: int             # of the measured pass
    parameter_bytes: int
    kept_bytes: int         # for the backward pass
    boundary_bytes: int     # the stream that the next layer reads
    all_to_all_bytes: int = 0   # that the tokens send to experts


def profile_layer(layer, tokens: int, repeats: int = 5, passes: int = 4) -> LayerProfile:
    """Medians over `repeats` of `passes` passes each, after one to warm up."""
    torch = layer.ops.torch
    given, dr = layer.sample(tokens)
    given = given if isinstance(given, tuple) else (given,)

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

    r, kept = layer.forward(*given)
    _, grads = layer.backward(dr, kept)
    return LayerProfile(forward=median(lambda: layer.forward(*given)), backward=median(lambda: layer.backward(dr, kept)),
                        update=median(lambda: layer.update(grads, 0.0)), tokens=tokens,
                        parameter_bytes=layer.parameter_bytes(), kept_bytes=layer.kept_bytes(kept),
                        boundary_bytes=r.numel() * r.element_size(), all_to_all_bytes=layer.all_to_all_bytes(tokens))


def measured_job(profiles, batch: int, seq: int = workloads.SEQ_LEN) -> dict:
    """A job for workloads.from_lists from its layers' profiles: times of the
    forward and backward pass scaled to a global batch of `batch` samples of
    `seq` tokens, bytes to one sample.  The speed-1 GPU is the one measured."""
    share = [seq / p.tokens for p in profiles]
    return dict(t=[(p.forward + p.backward) * s * batch for p, s in zip(profiles, share)],
                p=[p.parameter_bytes for p in profiles], a=[p.kept_bytes * s for p, s in zip(profiles, share)],
                x=[p.boundary_bytes * s for p, s in zip(profiles, share)],
                a2a=[p.all_to_all_bytes * s for p, s in zip(profiles, share)], batch=batch)


# one MI355X node: 288 GB a GPU, a 153 GB/s xGMI link between each two of its 8 GPUs, a
# 400 Gbit/s network link a GPU
MI355X = dict(speed=1.0, mem=288e9, bw_intra=153e9, bw_inter=50e9, gpus_per_node=8)


def main(argv=None) -> None:
    from . import arena
    ap = argparse.ArgumentParser(description="Times a model's layers on this GPU and estimates a job of them.")
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=0, help="default: 8/3 of --model, up to a multiple of 64")
    ap.add_argument("--layers", type=int, default=24)
    ap.add_argument("--experts", type=int, default=0, help="of every other layer; default: none has any")
    ap.add_argument("--choices", type=int, default=2, help="experts of a token")
    ap.add_argument("--vocabulary", type=int, default=0, help="of a loss behind the layers; default: there is none")
    ap.add_argument("--batch", type=int, default=128, help="global batch, samples")
    ap.add_argument("--samples", type=int, default=4, help="samples of the measured pass")
    ap.add_argument("--seq", type=int, default=workloads.SEQ_LEN)
    a = ap.parse_args(argv)
    inner = a.inner or -(-a.model * 8 // 3 // 64) * 64
    ops = LayerOps()
    kinds = {f"layer {a.model} x {inner}": lambda: FeedForwardLayer(ops, a.model, inner)}
    stack = [0] * a.layers
    if a.experts:
        kinds[f"layer of {a.experts} experts {a.model} x {inner}"] = \
            lambda: ExpertLayer(ops, a.model, inner, a.experts, a.choices)
        stack = [i % 2 for i in range(a.layers)]
    if a.vocabulary:
        stack.append(len(kinds))
        kinds[f"loss {a.model} x {a.vocabulary}"] = lambda: LossLayer(ops, a.model, a.vocabulary)
    profiles = []
    try:
        for name, make in kinds.items():
            p = profile_layer(make(), a.samples * a.seq)
            profiles.append(p)
            print(f"{name}, {p.tokens} tokens: forward {p.forward * 1e6:.1f} us, backward {p.backward * 1e6:.1f} us, "
                  f"update {p.update * 1e6:.1f} us; parameters {p.parameter_bytes / 1e6:.1f} MB, kept "
                  f"{p.kept_bytes / 1e6:.1f} MB, boundary {p.boundary_bytes / 1e6:.1f} MB, to experts "
                  f"{p.all_to_all_bytes / 1e6:.1f} MB", flush=True)
    finally:
        ops.torch.cuda.synchronize()
        ops.close()
    w = workloads.from_lists([measured_job([profiles[i] for i in stack], a.batch, a.seq)], [MI355X],
                             [1, 2, 4, 8, 16, 32], [1, 2, 4, 8, 16])
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
