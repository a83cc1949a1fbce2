"""The layer operators' definitions in 64 bits, for the tests: values, gradients
by the formulas, and elementwise bounds on what rounding in the operators may
change.

Bounds: u is half a unit in the last place at its largest share of the value
(8 bits of bfloat16: 2^-8, 11 of float16: 2^-11); a sum of K products in 32 bits is off by at most K 2^-23 of the
sum of magnitudes (whatever the order, with one unit for each product).
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}   # least subnormals


def act(z, name):
    """Value, derivative, and bounds of |first| and |second| derivative."""
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s), 1.1, 0.5
    if name == "gelu":
        c = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
        d = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return z * c, c + z * d, 1.13, 0.8
    return z.clamp_min(0), (z > 0).to(z.dtype), 1.0, 0.0


def ffn(x, wg, wu, wd, name, typ):
    """(y, bound), and what the gradients need."""
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    D, F = wg.shape[1], wg.shape[0]
    g, u = x @ wg.T, x @ wu.T
    dg, du = D * 2.0 ** -23 * (x.abs() @ wg.abs().T), D * 2.0 ** -23 * (x.abs() @ wu.abs().T)
    a, _, slope, _ = act(g, name)
    h = a * u
    bh = slope * dg * (u.abs() + du) + a.abs() * du + (U[typ] + 2.0 ** -20) * h.abs() + TINY[typ]
    y = h @ wd.T
    by = (bh + F * 2.0 ** -23 * h.abs()) @ wd.abs().T
    by = by * (1 + U[typ]) + U[typ] * y.abs() + TINY[typ]
    return y, by, dict(g=g, u=u, h=h, bg=dg, bu=du, bh=bh)


def ffn_back(dy, x, wg, wu, wd, name, typ, kept, grad_typ=None):
    """{name: (gradient, bound)} by the formulas."""
    dy, x, wg, wu, wd = (t.double() for t in (dy, x, wg, wu, wd))
    T, D, F = x.shape[0], x.shape[1], wg.shape[0]
    g, u, h = kept["g"], kept["u"], kept["h"]
    bg, bu = kept["bg"] + 2.0 ** -15 * g.abs(), kept["bu"] + 2.0 ** -15 * u.abs()      # kept in 24 bits
    a, d, slope, curve = act(g, name)
    jump = ((g.abs() <= bg) & (name == "relu")).double()       # the derivative's side is open there
    dh = dy @ wd
    bdh = D * 2.0 ** -23 * (dy.abs() @ wd.abs())
    du, dg = dh * a, dh * u * d
    bdu = bdh * (a.abs() + slope * bg) + dh.abs() * slope * bg + (U[typ] + 2.0 ** -20) * du.abs() + TINY[typ]
    bdg = ((bdh * (u.abs() + bu) + dh.abs() * bu) * (d.abs() + curve * bg + jump)
           + (dh * u).abs() * (curve * bg + jump) + (U[typ] + 2.0 ** -20) * dg.abs() + TINY[typ])
    out = {}

    def put(name, v, b, t):
        out[name] = v, b * (1 + U[t]) + U[t] * v.abs() + TINY[t]

    k2 = 2 * F * 2.0 ** -23
    put("dx", dg @ wg + du @ wu, (bdg + k2 * dg.abs()) @ wg.abs() + (bdu + k2 * du.abs()) @ wu.abs(), typ)
    gt, kt = grad_typ or typ, T * 2.0 ** -23
    put("dw_gate", dg.T @ x, (bdg + kt * dg.abs()).T @ x.abs(), gt)
    put("dw_up", du.T @ x, (bdu + kt * du.abs()).T @ x.abs(), gt)
    put("dw_down", dy.T @ h, dy.abs().T @ (kept["bh"] + kt * h.abs()), gt)
    return out


def norm(z, kind, eps):
    """Normalised rows, mean and 1 / deviation."""
    mu = z.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(z[:, :1])
    rs = 1 / torch.sqrt(((z - mu) ** 2).mean(1, keepdim=True) + eps)
    return (z - mu) * rs, mu, rs


def gate_of(gate, rows, tokens):
    if gate is None:
        return 1.0
    if not rows:
        return gate.double().reshape(1, -1)
    return gate.double()[torch.arange(tokens, device=gate.device) // rows]


def block(x, y, gate, rows, scale, w2, b2, w1, b1, kind, eps):
    """r and n of the fused norms; absent parameters None."""
    f = lambda t, v: v if t is None else t.double()
    r = x.double()
    if y is not None:
        v = norm(y.double(), kind, eps)[0] * f(w2, 1.0) + f(b2, 0.0)
        r = r + scale * gate_of(gate, rows, x.shape[0]) * v
    n = norm(r, kind, eps)[0] * f(w1, 1.0) + f(b1, 0.0)
    return r, n


def norm_back(q, zhat, rs, kind):
    m = (q * zhat).mean(1, keepdim=True)
    return rs * (q - zhat * m - (q.mean(1, keepdim=True) if kind == "layer" else 0))


def norm_back_size(q, zhat, rs, kind):
    """The magnitudes that norm_back adds up, q given by its magnitudes: what its rounding is relative to."""
    z = zhat.abs()
    return rs * (q + z * (q * z).mean(1, keepdim=True) + (q.mean(1, keepdim=True) if kind == "layer" else 0))


def block_back(dn, dr, r, y, stats, gate, rows, scale, w2, b2, w1, kind):
    """Gradients by the formulas from the stored r and the rows' statistics
    ([tokens][4]: mean and 1 / deviation of y, then of r); under "_name" the sums of
    the magnitudes that went into each."""
    f = lambda t, v: v if t is None else t.double()
    mag = lambda v: abs(v) if isinstance(v, float) else v.abs()
    s = stats.double()
    T = r.shape[0]
    out = {}
    d = torch.zeros_like(r, dtype=torch.float64) if dr is None else dr.double()
    size = d.abs()
    if dn is not None:
        rhat, dn = (r.double() - s[:, 2:3]) * s[:, 3:4], dn.double()
        # a value less its mean has lost what the two have in common
        z = (r.double().abs() + s[:, 2:3].abs()) * s[:, 3:4]
        d = d + norm_back(dn * f(w1, 1.0), rhat, s[:, 3:4], kind)
        size = size + norm_back_size((dn * f(w1, 1.0)).abs(), z, s[:, 3:4], kind)
        out["dw_pre"], out["db_pre"] = (dn * rhat).sum(0), dn.sum(0)
        out["_dw_pre"], out["_db_pre"] = (dn.abs() * z).sum(0), dn.abs().sum(0)
    out["dx"], out["_dx"] = d, size
    if y is not None:
        yhat, z = (y.double() - s[:, 0:1]) * s[:, 1:2], (y.double().abs() + s[:, 0:1].abs()) * s[:, 1:2]
        v, v_size = yhat * f(w2, 1.0) + f(b2, 0.0), z * mag(f(w2, 1.0)) + mag(f(b2, 0.0))
        g = scale * gate_of(gate, rows, T)
        dv, dv_size = g * d, mag(g) * size
        out["dy"] = norm_back(dv * f(w2, 1.0), yhat, s[:, 1:2], kind)
        out["_dy"] = norm_back_size(dv_size * mag(f(w2, 1.0)), z, s[:, 1:2], kind)
        out["dw_post"], out["db_post"] = (dv * yhat).sum(0), dv.sum(0)
        out["_dw_post"], out["_db_post"] = (dv_size * z).sum(0), dv_size.sum(0)
        if gate is not None:
            n = (gate.shape[0] if gate.dim() == 2 else 1) if rows else 1
            row = torch.arange(T, device=r.device) // rows if rows else torch.zeros(T, dtype=torch.long, device=r.device)
            for key, val in (("dgate", scale * d * v), ("_dgate", abs(scale) * size * v_size)):
                out[key] = torch.zeros(n, r.shape[1], dtype=torch.float64, device=r.device).index_add_(0, row, val)
    return out


def orthogonal(u, coefficients, steps, eps, scale):
    """The update of one matrix, from its (momentum's) value."""
    u = u.double()
    n = u.norm() + eps
    x = u / n if n > 0 else u
    flip = x.shape[0] > x.shape[1]
    x = x.T if flip else x
    for i in range(steps):
        a, b, c = coefficients[i] if hasattr(coefficients[0], "__len__") else coefficients
        m = x @ x.T
        x = a * x + b * (m @ x) + c * (m @ (m @ x))
    return scale * (x.T if flip else x)
