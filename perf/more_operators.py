"""Cases of the operators of a mixture-of-experts layer and of a language model's
last layer: the router, tokens sorted by expert and back, the experts' gated
blocks, and the cross entropy over a vocabulary, forward and backward.

The widths are those of the workloads (hidden sizes 1024, 2048 and 4096 of the
MoE jobs, sequences of 1024 tokens per sample); an expert's inner width is 8/3 of
the hidden size or, with many experts, a part of that.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
IGNORED = -100


def listed():
    return [
        # router: the one token of a running model, and a large batch with many experts
        {"name": "route one token", "op": "route", "train": False, "type": "bf16", "tokens": 1, "experts": 8, "k": 2,
         "normalise": True, "masked": 0.0},
        {"name": "route large", "op": "route", "train": True, "type": "f32", "tokens": 16384, "experts": 128, "k": 8,
         "normalise": True, "masked": 0.0},
        # tokens to experts and back: a few tokens of running sequences, odd sizes with
        # choices dropped, and a large microbatch with its gradients
        {"name": "sort few tokens", "op": "sort", "train": False, "type": "bf16", "tokens": 37, "model": 4096,
         "experts": 8, "k": 2, "dropped": 0.0},
        {"name": "sort odd", "op": "sort", "train": True, "type": "f16", "tokens": 3001, "model": 1365,
         "experts": 10, "k": 3, "dropped": 0.1},
        {"name": "sort large", "op": "sort", "train": True, "type": "bf16", "tokens": 16384, "model": 4096,
         "experts": 64, "k": 4, "dropped": 0.0},
        # experts' blocks: the two experts of one token, odd sizes on a few experts, many
        # narrow experts of a microbatch, eight wide ones of a large microbatch
        {"name": "experts one token", "op": "experts", "train": False, "type": "bf16", "act": "silu", "rows": 2,
         "model": 4096, "inner": 10944, "experts": 8, "spread": 0.5},
        {"name": "experts odd", "op": "experts", "train": True, "type": "f16", "act": "gelu", "rows": 1555,
         "model": 1000, "inner": 683, "experts": 7, "spread": 1.0},
        {"name": "experts many", "op": "experts", "train": True, "type": "bf16", "act": "silu", "rows": 16384,
         "model": 2048, "inner": 1408, "experts": 64, "spread": 0.5},
        {"name": "experts large", "op": "experts", "train": True, "type": "bf16", "act": "silu", "rows": 16384,
         "model": 4096, "inner": 10944, "experts": 8, "spread": 0.25},
        # loss: one scored token, odd sizes with ignored targets, a large microbatch
        {"name": "loss one token", "op": "loss", "train": False, "type": "bf16", "tokens": 1, "model": 4096,
         "vocabulary": 131072, "ignored": 0.0},
        {"name": "loss odd", "op": "loss", "train": True, "type": "f16", "tokens": 777, "model": 1000,
         "vocabulary": 50001, "ignored": 0.2},
        {"name": "loss large", "op": "loss", "train": True, "type": "bf16", "tokens": 8192, "model": 4096,
         "vocabulary": 131072, "ignored": 0.1},
    ]


def _size(rng, low, high, step=1):
    """A size spread evenly over its logarithm."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(low, min(high, v // step * step if v >= step else v))


def draw(rng):
    op = rng.choice(("route", "sort", "experts", "experts", "loss", "loss"))
    train = rng.random() < 0.6
    if op == "route":
        while True:
            c = {"op": op, "train": train, "type": rng.choice(("f32", "bf16", "f16")), "tokens": _size(rng, 1, 16384),
                 "experts": _size(rng, 2, 512), "k": rng.randint(1, 8), "normalise": rng.random() < 0.6,
                 "masked": rng.choice((0.0, 0.0, 0.3))}
            if c["k"] <= c["experts"] and c["tokens"] * c["experts"] <= 16384 * 128:
                return c
    if op == "sort":
        while True:
            c = {"op": op, "train": train, "type": rng.choice(("bf16", "f16", "f32")), "tokens": _size(rng, 1, 16384),
                 "model": _size(rng, 64, 8192, rng.choice((1, 64))), "experts": _size(rng, 2, 512),
                 "k": rng.randint(1, 8), "dropped": rng.choice((0.0, 0.0, 0.1))}
            if c["k"] <= c["experts"] and c["tokens"] * c["model"] * (c["k"] + 1) <= 16384 * 4096 * 4:
                return c
    step = rng.choice((1, 8, 64, 64))
    if op == "experts":
        while True:
            c = {"op": op, "train": train, "type": rng.choice(("bf16", "f16")), "act": rng.choice(("silu", "gelu")),
                 "rows": _size(rng, 1, 16384), "model": _size(rng, 256, 6144, step),
                 "inner": _size(rng, 128, 12288, step), "experts": _size(rng, 2, 128),
                 "spread": rng.choice((0.25, 0.5, 1.0))}
            weights = c["model"] * c["inner"]
            if c["experts"] * weights <= 8 * 4096 * 10944 and c["rows"] * weights <= 16384 * 4096 * 10944 // 4:
                return c
    while True:
        c = {"op": op, "train": train, "type": rng.choice(("bf16", "f16")), "tokens": _size(rng, 1, 8192),
             "model": _size(rng, 256, 6144, step), "vocabulary": _size(rng, 257, 131072, step),
             "ignored": rng.choice((0.0, 0.1))}
        if c["tokens"] * c["model"] * c["vocabulary"] <= 8192 * 4096 * 131072:
            return c


def prepare(case, seed):
    """Activations of unit variance, weights of standard deviation 1 / sqrt(fan in) (three times that in the
    vocabulary's, whose tokens' own rows the activations lean towards: a model that has learnt), experts of uneven
    popularity, gradients of a mean loss's size."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    typ = TYPES[case["type"]]

    def normal(shape, dtype=typ, std=1.0, mean=0.0):
        v = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
        return v.mul_(std).add_(mean).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda", dtype=torch.float32)

    s = dict(case)
    if case["op"] == "route":
        t, e, k = case["tokens"], case["experts"], case["k"]
        logits = normal((t, e), std=1.5)
        if case["masked"]:
            logits[uniform(t, e) < case["masked"]] = -math.inf
        s["logits"], s["scale"] = logits, 1.5
        if case["train"]:
            s["dweight"] = normal((t, k), torch.float32, 0.01)
    elif case["op"] == "sort":
        t, d, e, k = case["tokens"], case["model"], case["experts"], case["k"]
        scores = normal((t, e), torch.float32) + normal((e,), torch.float32, 0.5)
        value, index = torch.topk(scores, k, dim=1)
        s["index"] = torch.where(uniform(t, k) < case["dropped"], -1, index).to(torch.int32)
        s["weight"] = torch.softmax(value, 1)
        s["x"], s["ys"] = normal((t, d)), normal((t * k, d))
        s["xs"] = torch.zeros(t * k, d, dtype=typ, device="cuda")
        if case["train"]:
            s["dy"], s["dxs"] = normal((t, d), std=0.125), normal((t * k, d), std=0.125)
            s["dys"] = torch.zeros(t * k, d, dtype=typ, device="cuda")
    elif case["op"] == "experts":
        n, d, f, e = case["rows"], case["model"], case["inner"], case["experts"]
        popularity = torch.softmax(normal((e,), torch.float32, case["spread"]), 0)
        counts = torch.bincount(torch.multinomial(popularity, n, replacement=True, generator=gen), minlength=e)
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).to(torch.int32)
        s["most"] = int(counts.max())
        s["xs"] = normal((n, d))
        s["w_gate"], s["w_up"] = normal((e, f, d), std=d ** -0.5), normal((e, f, d), std=d ** -0.5)
        s["w_down"] = normal((e, d, f), std=f ** -0.5)
        if case["train"]:
            s["dys"] = normal((n, d), std=0.125)
    else:
        t, d, v = case["tokens"], case["model"], case["vocabulary"]
        target = torch.randint(0, v, (t,), generator=gen, device="cuda")
        s["w"] = normal((v, d), std=3 * d ** -0.5)
        s["x"] = (normal((t, d), torch.float32) + s["w"][target].float()).to(typ)
        s["target"] = torch.where(uniform(t) < case["ignored"], IGNORED, target)
        if case["train"]:
            s["dloss"] = uniform(t).add_(0.5).div_(t)
    return s


# ---------------------------------------------------------------- plain forms


def _route(s):
    """The k largest logits in order (of equal ones the first), their softmax, and the gradient of that."""
    l, k = s["logits"].float(), s["k"]
    value, index = torch.sort(l, dim=1, descending=True, stable=True)
    value, index = value[:, :k], index[:, :k]
    none = value == -math.inf
    m = l.amax(1, keepdim=True).clamp(min=-1e38)       # a row of nothing but -inf has no weights
    p = torch.exp(l - m)
    p = p / p.sum(1, keepdim=True).clamp(min=1e-30)
    q = torch.where(none, 0.0, p.gather(1, index))
    total = q.sum(1, keepdim=True).clamp(min=1e-30) if s["normalise"] else 1.0
    w = q / total
    out = {"index": torch.where(none, -1, index).to(torch.int32), "weight": s["scale"] * w}
    if s["train"]:
        dw = s["scale"] * s["dweight"]
        mean = (w * torch.where(none, 0.0, dw)).sum(1, keepdim=True)
        if s["normalise"]:
            dl = torch.zeros_like(l).scatter_(1, index, w * (dw - mean))
        else:
            dl = -p * mean
            dl = dl.scatter_add(1, index, torch.where(none, 0.0, q * dw))
        out["dlogits"] = dl.to(s["logits"].dtype)
    return out


def _sort(s):
    typ, k, e = s["x"].dtype, s["k"], s["experts"]
    t, d = s["x"].shape
    flat = s["index"].reshape(-1).long()
    kept = flat >= 0
    order = torch.argsort(torch.where(kept, flat, e), stable=True)         # dropped choices last
    counts = torch.zeros(e + 1, dtype=torch.int64, device="cuda").scatter_add_(0, torch.where(kept, flat, e),
                                                                              torch.ones_like(flat))
    offsets = torch.cat([torch.zeros_like(counts[:1]), counts[:e].cumsum(0)])
    row = torch.empty_like(flat).scatter_(0, order, torch.arange(t * k, device="cuda"))
    here = (torch.arange(t * k, device="cuda") < offsets[e])[:, None]
    xs = torch.where(here, s["x"][order // k], 0)
    each = torch.where(kept[:, None], s["ys"][row].float(), 0).view(t, k, d)
    w = torch.where(kept.view(t, k), s["weight"], 0)
    out = {"offsets": offsets.to(torch.int32), "row": torch.where(kept, row, -1).view(t, k).to(torch.int32), "xs": xs,
           "y": (w[:, :, None] * each).sum(1).to(typ)}
    if s["train"]:
        dy = s["dy"].float()
        dys = dy[order // k] * w.reshape(-1)[order][:, None]
        out["dys"] = torch.where(here, dys, 0).to(typ)
        out["dweight"] = (each * dy[:, None, :]).sum(2)
        out["dx"] = torch.where(kept[:, None], s["dxs"][row].float(), 0).view(t, k, d).sum(1).to(typ)
    return out


def _act(z, name):
    """The activation and its derivative."""
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    c = 0.5 * torch.erfc(z * -math.sqrt(0.5))
    return z * c, c + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _experts(s):
    """Experts side by side in one batched product: rows padded to the most that an expert has; of fewer rows than
    experts, the weights of each row's own."""
    typ, e = s["xs"].dtype, s["experts"]
    n, d = s["xs"].shape
    at = torch.arange(n, device="cuda")
    of = torch.searchsorted(s["offsets"].long(), at, right=True) - 1
    few = n <= e and not s["train"]
    cap, groups = (1, n) if few else (s["most"], e)
    place = at if few else of * cap + at - s["offsets"].long()[of]

    def padded(v):
        return torch.zeros(groups * cap, v.shape[1], device="cuda").index_copy_(0, place, v.float()).view(groups, cap, -1)

    def turned(v):
        return v.transpose(1, 2).contiguous()

    wg, wu, wd = ((s[k][of] if few else s[k]).float() for k in ("w_gate", "w_up", "w_down"))
    x = padded(s["xs"])
    g, u = torch.bmm(x, turned(wg)), torch.bmm(x, turned(wu))
    a, da = _act(g, s["act"])
    h = a * u
    out = {"ys": torch.bmm(h, turned(wd)).view(groups * cap, d)[place].to(typ)}
    if s["train"]:
        dy = padded(s["dys"])
        dh = torch.bmm(dy, wd)
        dg, du = dh * u * da, dh * a
        dxs = torch.bmm(dg, wg) + torch.bmm(du, wu)
        out.update(dxs=dxs.view(groups * cap, d)[place].to(typ), dw_gate=torch.bmm(turned(dg), x).to(typ),
                   dw_up=torch.bmm(turned(du), x).to(typ), dw_down=torch.bmm(turned(dy), h).to(typ))
    return out


def _loss(s):
    typ = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    l = x @ w.t()
    kept = s["target"] != IGNORED
    at = torch.where(kept, s["target"], 0)[:, None]
    m = l.amax(1, keepdim=True)
    p = torch.exp(l - m)
    total = p.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    out = {"loss": torch.where(kept, lse - l.gather(1, at)[:, 0], 0.0), "lse": lse}
    if s["train"]:
        dl = torch.where(kept, s["dloss"], 0.0)[:, None]
        g = p * (dl / total)
        g.scatter_add_(1, at, -dl)
        out.update(dx=(g @ w).to(typ), dw=(g.t() @ x).to(typ))
    return out


_kept = {}


def run(s):
    if not own:
        return {"route": _route, "sort": _sort, "experts": _experts, "loss": _loss}[s["op"]](s)
    if "ops" not in _kept:
        from paper_2403_16125_amd.layer import LayerOps
        _kept["ops"] = LayerOps()
    ops = _kept["ops"]
    if s["op"] == "route":
        index, weight = ops.route(s["logits"], s["k"], normalise=s["normalise"], scale=s["scale"])
        out = {"index": index, "weight": weight}
        if s["train"]:
            out["dlogits"] = ops.route_backward(s["dweight"], s["logits"], index, normalise=s["normalise"],
                                                scale=s["scale"])
        return out
    if s["op"] == "sort":
        plan = ops.sort_by_expert(s["index"], s["experts"])
        xs = ops.dispatch(s["x"], plan, out=s["xs"])
        out = {"offsets": plan.offsets, "row": plan.row, "xs": xs, "y": ops.combine(s["ys"], plan, s["weight"])}
        if s["train"]:
            out["dys"], out["dweight"] = ops.combine_backward(s["dy"], s["ys"], plan, s["weight"], out=s["dys"])
            out["dx"] = ops.dispatch_backward(s["dxs"], plan)
        return out
    if s["op"] == "experts":
        weights = (s["w_gate"], s["w_up"], s["w_down"])
        if not s["train"]:
            return {"ys": ops.experts_forward(s["xs"], s["offsets"], *weights, activation=s["act"])}
        ys, saved = ops.experts_forward(s["xs"], s["offsets"], *weights, activation=s["act"], save=True)
        dxs, dw_gate, dw_up, dw_down = ops.experts_backward(s["dys"], s["xs"], s["offsets"], *weights, saved,
                                                            activation=s["act"])
        return {"ys": ys, "dxs": dxs, "dw_gate": dw_gate, "dw_up": dw_up, "dw_down": dw_down}
    loss, lse = ops.cross_entropy_forward(s["x"], s["w"], s["target"], ignore_index=IGNORED)
    out = {"loss": loss, "lse": lse}
    if s["train"]:
        out["dx"], out["dw"] = ops.cross_entropy_backward(s["dloss"], s["x"], s["w"], s["target"], lse,
                                                          ignore_index=IGNORED)
    return out


def work(case):
    """Each input read once, each output written once.  Of the experts' weights only those of experts that can have
    rows; a loss whose logits are not kept forms them in both directions."""
    b = {"f32": 4, "bf16": 2, "f16": 2}[case["type"]]
    train = case["train"]
    if case["op"] == "route":
        t, e, k = case["tokens"], case["experts"], case["k"]
        return {"bytes": t * (e * b + 8 * k) + (t * (e * b + 4 * k) if train else 0), "flops": t * e * (12 if train else 6)}
    if case["op"] == "sort":
        t, d, k = case["tokens"], case["model"], case["k"]
        moved = b * t * d * (1 + k + k + 1) + 12 * t * k
        return {"bytes": moved + (b * t * d * (1 + k + k + 1) + 4 * t * k if train else 0),
                "flops": t * k * d * (6 if train else 2)}
    if case["op"] == "experts":
        n, d, f = case["rows"], case["model"], case["inner"]
        e = min(case["experts"], n) if not train else case["experts"]
        if not train:
            return {"bytes": b * (2 * n * d + 3 * e * d * f), "flops": 6 * n * d * f}
        return {"bytes": b * (4 * n * d + 6 * e * d * f), "flops": 18 * n * d * f}
    t, d, v = case["tokens"], case["model"], case["vocabulary"]
    if not train:
        return {"bytes": b * (t * d + v * d) + 16 * t, "flops": 2 * t * d * v}
    return {"bytes": 2 * b * (t * d + v * d) + 20 * t, "flops": 8 * t * d * v}


# ------------------------------------------------------- 64-bit definitions


def _exact_route(s):
    """Weights by the definition over the chosen logits, gradients by differentiating it."""
    logits = s["logits"].double().requires_grad_(s["train"])
    order = torch.argsort(s["logits"].double(), dim=1, descending=True, stable=True)[:, :s["k"]]
    taken = torch.gather(logits, 1, order)
    there = taken.detach() > -math.inf
    over = taken if s["normalise"] else logits
    live = over.detach() > -math.inf
    over = torch.where(live, over, torch.zeros_like(over))
    top = torch.where(live, over.detach(), torch.full_like(over, -1e300)).amax(1, keepdim=True).clamp(min=-1e299)
    whole = (torch.exp(over - top) * live).sum(1, keepdim=True)
    taken = torch.where(there, taken, torch.zeros_like(taken))
    weight = s["scale"] * torch.exp(taken - top) * there / torch.where(whole > 0, whole, torch.ones_like(whole))
    out = {"index": None, "weight": weight.detach()}
    if s["train"]:
        out["dlogits"] = torch.autograd.grad((weight * s["dweight"].double()).sum(), logits)[0]
    return out


def _exact_sort(s):
    """Choice by choice through the positions that a sort of (expert, place) gives."""
    t, k = s["index"].shape
    flat = s["index"].reshape(-1).long()
    choice = torch.nonzero(flat >= 0).flatten()
    choice = choice[torch.argsort(flat[choice] * (t * k) + choice)]
    token, n = torch.div(choice, k, rounding_mode="floor"), choice.numel()
    weight = s["weight"].double().reshape(-1)[choice][:, None]
    ys = s["ys"].double()[:n]
    out = {"offsets": None, "row": None, "xs": torch.zeros_like(s["xs"], dtype=torch.float64)}
    out["xs"][:n] = s["x"].double()[token]
    out["y"] = torch.zeros_like(s["x"], dtype=torch.float64).index_add_(0, token, weight * ys)
    if s["train"]:
        dy = s["dy"].double()[token]
        out["dys"] = torch.zeros_like(s["dys"], dtype=torch.float64)
        out["dys"][:n] = weight * dy
        out["dweight"] = torch.zeros(t * k, dtype=torch.float64, device="cuda")
        out["dweight"][choice] = (ys * dy).sum(1)
        out["dweight"] = out["dweight"].view(t, k)
        out["dx"] = torch.zeros_like(s["x"], dtype=torch.float64).index_add_(0, token, s["dxs"].double()[:n])
    return out


def _exact_experts(s):
    bounds, parts = s["offsets"].tolist(), []
    for i in range(s["experts"]):
        rows = slice(bounds[i], bounds[i + 1])
        x, (wg, wu, wd) = s["xs"][rows].double(), (s[k][i].double() for k in ("w_gate", "w_up", "w_down"))
        g, u = torch.mm(x, wg.T), torch.mm(x, wu.T)
        if s["act"] == "silu":
            e = 1 / (1 + torch.exp(-g))
            a, da = g * e, e + g * e * (1 - e)
        else:
            phi = torch.special.ndtr(g)
            a, da = g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        part = {"ys": torch.mm(a * u, wd.T)}
        if s["train"]:
            dy = s["dys"][rows].double()
            dh = torch.mm(dy, wd)
            dg, du = dh * u * da, dh * a
            part.update(dxs=torch.mm(dg, wg) + torch.mm(du, wu), dw_gate=torch.mm(dg.T, x), dw_up=torch.mm(du.T, x),
                        dw_down=torch.mm(dy.T, a * u))
        parts.append(part)
    return {k: (torch.cat if k in ("ys", "dxs") else torch.stack)([p[k] for p in parts]) for k in parts[0]}


def _exact_loss(s):
    """Token by token in blocks, so that the logits in 64 bits stay small."""
    x, w = s["x"].double(), s["w"].double()
    n, step = x.shape[0], 1024
    loss, lse, dx, dw = [], [], [], torch.zeros_like(w) if s["train"] else None
    for i in range(0, n, step):
        rows = slice(i, min(n, i + step))
        logits, target = torch.mm(x[rows], w.T), s["target"][rows]
        norm = torch.logsumexp(logits, 1)
        at = torch.nonzero(target != IGNORED).flatten()
        value = torch.zeros_like(norm)
        value[at] = norm[at] - logits[at, target[at]]
        loss.append(value)
        lse.append(norm)
        if s["train"]:
            dl = torch.zeros_like(norm)
            dl[at] = s["dloss"][rows].double()[at]
            g = torch.exp(logits - norm[:, None])
            g[at, target[at]] -= 1
            g *= dl[:, None]
            dx.append(torch.mm(g, w))
            dw += torch.mm(g.T, x[rows])
    out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    if s["train"]:
        out.update(dx=torch.cat(dx), dw=dw)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "sort": _exact_sort, "experts": _exact_experts, "loss": _exact_loss}[case["op"]](s)
