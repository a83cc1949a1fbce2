"""The layer operators on the GPU against their definitions in 64 bits.

Feed-forward: elementwise bounds derived in layer_reference.  Norms: one
rounding to the output's type (u |v|) beside, for the 32-bit arithmetic, 2^-17 of
the row's size (forward) or of the magnitudes that a gradient adds up.  Orthogonalised
update: 1e-2 of the result's norm: five steps, each rounding three matrices to
2^-11 relative at most, taken a few times larger by the polynomials, and the
result's own rounding.
"""
import ctypes

import pytest
import torch

import layer_reference as ref
from paper_2403_16125_amd import arena, layer

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
COEF = layer.COEFFICIENTS


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    yield o
    torch.cuda.synchronize()
    o.close()


def normal(shape, dtype, seed, std=1.0, mean=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)


def inside(name, got, want, bound):
    off = (got.double() - want).abs() - bound
    at = int(off.argmax())
    assert off.max() <= 0 and not torch.isnan(got).any(), \
        f"{name}: {got.reshape(-1)[at].item()} for {want.reshape(-1)[at].item()}, bound {bound.reshape(-1)[at].item()}"


def strided(t, pad, offset):
    """t in rows of `pad` more values, starting `offset` values into the memory; NaN around it."""
    rows, cols = t.shape
    mem = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=t.dtype, device=t.device)
    v = mem[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


# ---------------------------------------------------------------- feed-forward

def ffn_inputs(T, D, F, typ, seed=1):
    return (normal((T, D), typ, seed), normal((F, D), typ, seed + 1, D ** -0.5), normal((F, D), typ, seed + 2, D ** -0.5),
            normal((D, F), typ, seed + 3, F ** -0.5), normal((T, D), typ, seed + 4, 0.25))


def check_ffn(ops, t, act, typ, back=True):
    x, wg, wu, wd, dy = t
    y, saved = ops.ffn_forward(x, wg, wu, wd, activation=act, save=True)
    only = ops.ffn_forward(x, wg, wu, wd, activation=act)
    want, bound, kept = ref.ffn(x, wg, wu, wd, act, typ)
    inside("y", y, want, bound)
    assert torch.equal(y, only)
    if back:
        got = ops.ffn_backward(dy, x, wg, wu, wd, saved, activation=act)
        for (name, (v, b)), g in zip(ref.ffn_back(dy, x, wg, wu, wd, act, typ, kept).items(), got):
            inside(name, g, v, b)


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T,D,F", [(1, 64, 96), (3, 1, 1), (16, 40, 24), (17, 129, 63), (32, 256, 40), (33, 72, 515),
                                   (64, 128, 128), (65, 128, 128), (130, 200, 328), (257, 257, 257), (300, 136, 1000)])
def test_ffn(ops, T, D, F, act, typ):
    check_ffn(ops, ffn_inputs(T, D, F, typ), act, typ)


@pytest.mark.parametrize("T,D,F", [(1024, 1024, 2752), (2048, 512, 1376), (777, 1000, 2731), (40, 2048, 5504),
                                   (1, 4096, 10944), (96, 4096, 1368), (5000, 64, 128)])
def test_ffn_larger(ops, T, D, F):
    check_ffn(ops, ffn_inputs(T, D, F, BF16), "silu", BF16)


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("pad,offset", [(0, 1), (8, 0), (3, 0), (24, 8), (1, 5)])
def test_ffn_strides_and_alignment(ops, T, pad, offset):
    """Rows apart by more than their width, memory that starts on any value, NaN between the rows."""
    t = [strided(v, pad, offset) for v in ffn_inputs(T, 96, 168, BF16)]
    check_ffn(ops, t, "silu", BF16)
    # the gate and up weights with strides of their own
    t[1] = strided(t[1], 16, 0)
    check_ffn(ops, t, "silu", BF16)


@pytest.mark.parametrize("T", [7, 100])
def test_ffn_outputs_keep_to_their_rows(ops, T):
    x, wg, wu, wd, dy = ffn_inputs(T, 72, 56, F16)
    y0, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    mem = torch.full((T + 2, 80), 7.0, dtype=F16, device="cuda")
    ops.ffn_forward(x, wg, wu, wd, out=mem[1:-1, 3:75])
    assert torch.equal(mem[1:-1, 3:75], y0)
    mem[1:-1, 3:75] = 7.0
    assert bool((mem == 7.0).all())
    want = ops.ffn_backward(dy, x, wg, wu, wd, saved)
    boxes = [torch.full((r + 2, c + 9), 7.0, dtype=F16, device="cuda") for r, c in ((56, 72), (56, 72), (72, 56))]
    views = [b[1:-1, 5:-4] for b in boxes]
    got = ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=views)
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    for b, v in zip(boxes, views):
        v.fill_(7.0)
        assert bool((b == 7.0).all())


@pytest.mark.parametrize("typ", [BF16, F16])
@pytest.mark.parametrize("T,D,F", [(130, 200, 328), (20, 65, 33)])
def test_ffn_float_gradients_accumulate(ops, T, D, F, typ):
    x, wg, wu, wd, dy = ffn_inputs(T, D, F, typ)
    _, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    _, _, kept = ref.ffn(x, wg, wu, wd, "silu", typ)
    want = ref.ffn_back(dy, x, wg, wu, wd, "silu", typ, kept, F32)
    grads = [torch.full(w.shape, 0.5, device="cuda") for w in (wg, wu, wd)]
    first = ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=[torch.empty_like(g) for g in grads])[1:]
    got = ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=grads, accumulate=True)[1:]
    for name, f, g in zip(("dw_gate", "dw_up", "dw_down"), first, got):
        v, b = want[name]
        inside(name, f, v, b)
        inside(name + " + 0.5", g, f.double() + 0.5, (f.double() + 0.5).abs() * 2.0 ** -24)


def test_ffn_no_tokens(ops):
    x, wg, wu, wd, dy = ffn_inputs(0, 64, 96, BF16)
    y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    assert y.shape == (0, 64)
    dx, *grads = ops.ffn_backward(dy, x, wg, wu, wd, saved)
    assert dx.shape == (0, 64) and all(bool((g == 0).all()) for g in grads)
    kept = [torch.ones_like(g) for g in grads]
    ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=kept, accumulate=True)
    assert all(bool((g == 1).all()) for g in kept)


@pytest.mark.parametrize("T", [9, 140])
def test_ffn_bad_values_stay_in_their_row(ops, T):
    x, wg, wu, wd, _ = ffn_inputs(T, 64, 80, BF16)
    y0 = ops.ffn_forward(x, wg, wu, wd)
    x = x.clone()
    x[4], x[7, 3] = float("inf"), float("nan")
    y = ops.ffn_forward(x, wg, wu, wd)
    good = [i for i in range(T) if i not in (4, 7)]
    assert torch.equal(y[good], y0[good])
    assert not torch.isfinite(y[4]).any() and torch.isnan(y[7]).all()


def test_ffn_extreme_gates(ops):
    """Gates far past where exp overflows: silu(z) = 0 below, z above."""
    D = F = 16
    x = torch.zeros(2, D, dtype=BF16, device="cuda")
    x[0, 0], x[1, 0] = 1.0, -1.0
    wg = torch.zeros(F, D, dtype=BF16, device="cuda")
    wg[:, 0] = 1e4
    wu = torch.zeros_like(wg)
    wu[:, 0] = 1.0
    y, saved = ops.ffn_forward(x, wg, wu, torch.eye(D, dtype=BF16, device="cuda"), save=True)
    assert bool((y[0] == 9984.0).all()) and bool((y[1] == 0).all())     # 1e4 in bfloat16
    got = ops.ffn_backward(torch.ones_like(x), x, wg, wu, torch.eye(D, dtype=BF16, device="cuda"), saved)
    assert all(bool(torch.isfinite(g).all()) for g in got)


# ---------------------------------------------------------------- norms

def norm_inputs(T, D, typ, stream, rows, seed=3):
    groups = -(-T // rows) if rows else 1
    return dict(x=normal((T, D), stream, seed, 2.0), y=normal((T, D), typ, seed + 1, 0.7, 0.1),
                gate=normal((groups, D), typ, seed + 2, 0.3, 0.5), w_post=normal((D,), typ, seed + 3, 0.1, 1.0),
                b_post=normal((D,), typ, seed + 4, 0.1), w_pre=normal((D,), typ, seed + 5, 0.1, 1.0),
                b_pre=normal((D,), typ, seed + 6, 0.1), dn=normal((T, D), typ, seed + 7, 0.3),
                dr=normal((T, D), stream, seed + 8, 0.3))


def near_rows(name, got, want):
    size = (want ** 2).mean(-1, keepdim=True).sqrt() + want.abs().amax(-1, keepdim=True)
    inside(name, got, want, ref.U[got.dtype] * want.abs() + 2.0 ** -17 * size + ref.TINY[got.dtype])


def near_sums(name, got, want, size):
    inside(name, got, want, ref.U[got.dtype] * want.abs() + 2.0 ** -17 * size + ref.TINY[got.dtype])


def check_norm(ops, t, rows, kind, scale=0.5, eps=1e-5, use=("gate", "w_post", "b_post", "w_pre", "b_pre")):
    p = {k: t[k] if k in use else None for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
    given = dict(p, gate_rows=rows, scale=scale, kind=kind, eps=eps)
    r, n, stats = ops.norm_forward(t["x"], t["y"], save=True, **given)
    r2, n2 = ops.norm_forward(t["x"], t["y"], **given)
    assert torch.equal(r, r2) and torch.equal(n, n2)
    wr, wn = ref.block(t["x"], t["y"], p["gate"], rows, scale, p["w_post"], p["b_post"], p["w_pre"], p["b_pre"], kind, eps)
    near_rows("r", r, wr)
    near_rows("n", n, wn)
    got = ops.norm_backward(t["dn"], t["dr"], r, t["y"], stats, **given)
    want = ref.block_back(t["dn"], t["dr"], r, t["y"], stats, p["gate"], rows, scale, p["w_post"], p["b_post"],
                          p["w_pre"], kind)
    near_sums("dx", got["dx"], want["dx"], want["_dx"])
    near_sums("dy", got["dy"], want["dy"], want["_dy"])
    for k in p:
        if p[k] is not None:
            near_sums("d" + k, got["d" + k], want["d" + k].reshape(p[k].shape), want["_d" + k].reshape(p[k].shape))
        else:
            assert got["d" + k] is None


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("typ,stream", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, F32)])
@pytest.mark.parametrize("T,D,rows", [(1, 1, 0), (1, 513, 0), (5, 64, 2), (7, 511, 1), (300, 512, 100), (33, 1365, 0),
                                      (17, 2048, 16), (700, 2049, 256), (6, 4096, 4), (9, 8191, 0), (5, 16384, 3)])
def test_norm(ops, T, D, rows, typ, stream, kind):
    if D == 1 and kind == "layer":
        return          # one value less its own mean: nothing is left to compare
    check_norm(ops, norm_inputs(T, D, typ, stream, rows), rows, kind)


@pytest.mark.parametrize("use", [(), ("gate",), ("w_post", "w_pre"), ("b_pre",), ("b_post", "gate")])
def test_norm_without_parameters(ops, use):
    check_norm(ops, norm_inputs(20, 200, BF16, BF16, 0), 0, "rms", use=use)


@pytest.mark.parametrize("typ,stream", [(BF16, BF16), (F16, F32), (F32, F32)])
@pytest.mark.parametrize("T,D", [(50, 1500), (9, 3000), (700, 5000), (40, 8000), (600, 9000)])
def test_norm_without_biases(ops, T, D, typ, stream):
    """The rows' shapes by width, where two fewer sums leave other forms of the backward."""
    check_norm(ops, norm_inputs(T, D, typ, stream, 300), 300, "rms", use=("gate", "w_post", "w_pre"))


@pytest.mark.parametrize("T,D,rows", [(4100, 512, 1000), (3001, 520, 7), (2500, 96, 1), (1500, 3000, 600)])
def test_norm_gate_rows_across_workers(ops, T, D, rows):
    """Gate rows shared by workers, several to a worker, one token each."""
    check_norm(ops, norm_inputs(T, D, F32, F32, rows), rows, "layer")


def test_norm_before_only_and_after_only(ops):
    t = norm_inputs(30, 300, BF16, F32, 0)
    r, n, stats = ops.norm_forward(t["x"], w_pre=t["w_pre"], dtype=BF16, save=True)
    assert r is t["x"] and n.dtype == BF16
    near_rows("n", n, ref.block(t["x"], None, None, 0, 1.0, None, None, t["w_pre"], None, "rms", 1e-6)[1])
    got = ops.norm_backward(t["dn"], None, r, None, stats, w_pre=t["w_pre"])
    want = ref.block_back(t["dn"], None, r, None, stats, None, 0, 1.0, None, None, t["w_pre"], "rms")
    near_sums("dx", got["dx"], want["dx"], want["_dx"])
    near_sums("dw_pre", got["dw_pre"], want["dw_pre"], want["_dw_pre"])
    r, n, stats = ops.norm_forward(t["x"], t["y"], w_post=t["w_post"], next_norm=False, save=True)
    assert n is None
    near_rows("r", r, ref.block(t["x"], t["y"], None, 0, 1.0, t["w_post"], None, None, None, "rms", 1e-6)[0])
    got = ops.norm_backward(None, t["dr"], r, t["y"], stats, w_post=t["w_post"])
    want = ref.block_back(None, t["dr"], r, t["y"], stats, None, 0, 1.0, t["w_post"], None, None, "rms")
    assert torch.equal(got["dx"], t["dr"])
    near_sums("dy", got["dy"], want["dy"], want["_dy"])


@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 0), (8, 8), (1, 5)])
@pytest.mark.parametrize("D", [96, 700, 2050])
def test_norm_strides_and_alignment(ops, D, pad, offset):
    t = norm_inputs(11, D, BF16, F32, 4)
    for k in ("x", "y", "gate", "dn", "dr"):
        t[k] = strided(t[k], pad, offset)
    for k in ("w_post", "b_post", "w_pre", "b_pre"):
        t[k] = strided(t[k].view(1, -1), 0, offset)[0]
    check_norm(ops, t, 4, "layer")


def test_norm_zero_rows_and_no_tokens(ops):
    t = norm_inputs(6, 128, BF16, BF16, 0)
    t["x"][2], t["y"][2], t["y"][3] = 0, 0, 0
    check_norm(ops, t, 0, "rms")
    x, y = t["x"][:0], t["y"][:0]
    r, n, stats = ops.norm_forward(x, y, gate=t["gate"], w_pre=t["w_pre"], save=True)
    assert r.shape == n.shape == (0, 128)
    got = ops.norm_backward(n, r, r, y, stats, gate=t["gate"], w_pre=t["w_pre"])
    assert got["dx"].shape == (0, 128) and bool((got["dgate"] == 0).all()) and bool((got["dw_pre"] == 0).all())
    # no eps: a row of zeros has no direction, and only that row
    r, n = ops.norm_forward(t["x"], eps=0.0)
    assert torch.isnan(n[2]).all() and torch.isfinite(n[:2]).all()


def test_norm_bad_values_stay_in_their_row(ops):
    t = norm_inputs(8, 600, BF16, F32, 0)
    given = dict(gate=t["gate"], w_post=t["w_post"], w_pre=t["w_pre"])
    r0, n0 = ops.norm_forward(t["x"], t["y"], **given)
    t["y"][3, 5], t["x"][6, 1] = float("inf"), float("nan")
    r, n = ops.norm_forward(t["x"], t["y"], **given)
    good = [0, 1, 2, 4, 5, 7]
    assert torch.equal(r[good], r0[good]) and torch.equal(n[good], n0[good])
    assert torch.isnan(n[3]).any() and torch.isnan(n[6]).all()


def test_norm_large_mean(ops):
    """A mean a thousand times the deviation: squares are taken about the mean."""
    x = normal((50, 1000), F32, 5, 1.0, 1000.0)
    _, n = ops.norm_forward(x, kind="layer")
    want = ref.norm(x.double(), "layer", 1e-6)[0]
    inside("n", n, want, torch.full_like(want, 1000 * 2.0 ** -22))


def test_norm_wide_rows_in_place(ops):
    """Past 8192 columns the sums have a pass of their own, which then finds dx where dr was."""
    T, D = 30, 9000
    t = norm_inputs(T, D, BF16, F32, 7)
    given = dict(gate=t["gate"], gate_rows=7, w_post=t["w_post"], w_pre=t["w_pre"], scale=0.5)
    r, n, stats = ops.norm_forward(t["x"], t["y"], save=True, **given)
    want = ops.norm_backward(t["dn"], t["dr"], r, t["y"], stats, **given)
    dr = t["dr"].clone()
    dgate, dw2, dw1 = torch.empty_like(t["gate"]), torch.empty_like(t["w_post"]), torch.empty_like(t["w_pre"])
    d = layer.NormDesc(dtype=1, stream_dtype=0, kind=0, width=D, tokens=T, gate_rows=7, eps=1e-6, scale=0.5,
                       y=t["y"].data_ptr(), ld_y=D, gate=t["gate"].data_ptr(), ld_gate=D, w_post=t["w_post"].data_ptr(),
                       w_pre=t["w_pre"].data_ptr(), r=r.data_ptr(), ld_r=D, stats=stats.data_ptr())
    need = layer.arena_norm_backward_workspace(ops.ctx, d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = layer.NormGrads(dn=t["dn"].data_ptr(), ld_dn=D, dr=dr.data_ptr(), ld_dr=D, dx=dr.data_ptr(), ld_dx=D,
                        dgate=dgate.data_ptr(), dw_post=dw2.data_ptr(), dw_pre=dw1.data_ptr(), workspace=ws.data_ptr(),
                        workspace_bytes=need)
    layer.arena_norm_backward(ops.ctx, d, g, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(dr, want["dx"])
    sizes = ref.block_back(t["dn"], t["dr"], r, t["y"], stats, t["gate"], 7, 0.5, t["w_post"], None, t["w_pre"], "rms")
    for name, got in (("dgate", dgate), ("dw_post", dw2), ("dw_pre", dw1)):
        near_sums(name, got, sizes[name], sizes["_" + name])


def test_norm_many_rows(ops):
    """More rows than a launch's workers."""
    x = normal((4200000, 6), BF16, 12)
    r, n = ops.norm_forward(x, x, kind="layer", eps=1e-3)
    wr, wn = ref.block(x, x, None, 0, 1.0, None, None, None, None, "layer", 1e-3)
    near_rows("r", r, wr)
    near_rows("n", n, wn)


@pytest.mark.parametrize("T", [3, 40])
def test_ffn_gate_and_up_with_strides_of_their_own(ops, T):
    x, wg, wu, wd, dy = ffn_inputs(T, 64, 96, BF16)
    check_ffn(ops, (x, strided(wg, 8, 0), strided(wu, 24, 8), wd, dy), "gelu", BF16)


def test_norm_in_place(ops):
    """r over x and dx over dr, as the header allows."""
    t = norm_inputs(40, 520, BF16, F32, 0)
    r, n, stats = ops.norm_forward(t["x"], t["y"], save=True)
    x = t["x"].clone()
    n2 = torch.empty_like(n)
    stream = torch.cuda.current_stream().cuda_stream
    d = layer.NormDesc(dtype=1, stream_dtype=0, kind=0, width=520, tokens=40, eps=1e-6, scale=1.0, x=x.data_ptr(), ld_x=520,
                       y=t["y"].data_ptr(), ld_y=520, r=x.data_ptr(), ld_r=520, n=n2.data_ptr(), ld_n=520,
                       stats=stats.data_ptr())
    layer.arena_norm_forward(ops.ctx, d, stream)
    assert torch.equal(x, r) and torch.equal(n2, n)
    want = ops.norm_backward(t["dn"], t["dr"], r, t["y"], stats)
    dr = t["dr"].clone()
    need = layer.arena_norm_backward_workspace(ops.ctx, d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = layer.NormGrads(dn=t["dn"].data_ptr(), ld_dn=520, dr=dr.data_ptr(), ld_dr=520, dx=dr.data_ptr(), ld_dx=520,
                        workspace=ws.data_ptr(), workspace_bytes=need)
    layer.arena_norm_backward(ops.ctx, d, g, stream)
    assert torch.equal(dr, want["dx"])


@pytest.mark.parametrize("D", [2, 5, 7, 8, 9, 15, 505, 513, 519, 1366, 2047, 2053, 4099, 8197, 9001])
def test_norm_rows_of_all_ends(ops, D):
    """Rows that end inside eight values: what lies past them is neither used nor written, in place or not."""
    T, gap = 21, 11
    t = norm_inputs(T, D, BF16, F32, 0)
    given = dict(gate=t["gate"], w_post=t["w_post"], w_pre=t["w_pre"], scale=0.5, kind="layer", eps=1e-3)
    r, n, stats = ops.norm_forward(t["x"], t["y"], save=True, **given)
    want = ops.norm_backward(t["dn"], t["dr"], r, t["y"], stats, **given)

    def wide(v, fill):
        w = torch.full((T, D + gap), fill, dtype=v.dtype, device="cuda")
        w[:, :D] = v
        return w
    nan = float("nan")
    x, y, dn, dr = wide(t["x"], nan), wide(t["y"], nan), wide(t["dn"], nan), wide(t["dr"], nan)
    n2 = wide(torch.zeros_like(n), 7.0)
    s2 = torch.empty_like(stats)
    dw2, dw1 = torch.empty_like(t["w_post"]), torch.empty_like(t["w_pre"])
    dgate = torch.empty_like(t["gate"])
    stream, L = torch.cuda.current_stream().cuda_stream, D + gap
    d = layer.NormDesc(dtype=1, stream_dtype=0, kind=1, width=D, tokens=T, eps=1e-3, scale=0.5, x=x.data_ptr(), ld_x=L,
                       y=y.data_ptr(), ld_y=L, gate=t["gate"].data_ptr(), ld_gate=D, w_post=t["w_post"].data_ptr(),
                       w_pre=t["w_pre"].data_ptr(), r=x.data_ptr(), ld_r=L, n=n2.data_ptr(), ld_n=L, stats=s2.data_ptr())
    layer.arena_norm_forward(ops.ctx, d, stream)
    assert torch.equal(x[:, :D], r) and bool(x[:, D:].isnan().all())
    assert torch.equal(n2[:, :D], n) and bool((n2[:, D:] == 7.0).all()) and torch.equal(s2, stats)
    need = layer.arena_norm_backward_workspace(ops.ctx, d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dy = wide(torch.zeros_like(t["y"]), 7.0)
    g = layer.NormGrads(dn=dn.data_ptr(), ld_dn=L, dr=dr.data_ptr(), ld_dr=L, dx=dr.data_ptr(), ld_dx=L,
                        dy=dy.data_ptr(), ld_dy=L, dgate=dgate.data_ptr(), dw_post=dw2.data_ptr(),
                        dw_pre=dw1.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=need)
    layer.arena_norm_backward(ops.ctx, d, g, stream)
    assert torch.equal(dr[:, :D], want["dx"]) and bool(dr[:, D:].isnan().all())
    assert torch.equal(dy[:, :D], want["dy"]) and bool((dy[:, D:] == 7.0).all())
    sizes = ref.block_back(t["dn"], t["dr"], r, t["y"], stats, t["gate"], 0, 0.5, t["w_post"], None, t["w_pre"], "layer")
    for name, got in (("dgate", dgate), ("dw_post", dw2), ("dw_pre", dw1)):
        near_sums(name, got, sizes[name].reshape(got.shape), sizes["_" + name].reshape(got.shape))


# ---------------------------------------------------------------- orthogonalised update

def check_update(ops, grad, steps=5, coefficients=COEF, scale=1.5, momentum=None, mu=0.9, nesterov=True, dtype=BF16,
                 eps=1e-7):
    stack = grad if grad.dim() == 3 else grad[None]
    u, m = stack.double(), None
    if momentum is not None:
        m = mu * (momentum if momentum.dim() == 3 else momentum[None]).double() + u
        u = u + mu * m if nesterov else m
    kept = None if momentum is None else momentum.clone()
    got = ops.orthogonal_update(grad, momentum=kept, mu=mu, nesterov=nesterov, coefficients=coefficients, steps=steps,
                                eps=eps, scale=scale, dtype=dtype)
    if m is not None:
        size = mu * momentum.double().abs() + grad.double().abs()       # what the sum may cancel
        inside("momentum", kept, m.reshape(kept.shape), 2.0 ** -22 * size)
    for g, v in zip(got if got.dim() == 3 else got[None], u):
        want = ref.orthogonal(v, coefficients, steps, eps, scale)
        assert (g.double() - want).norm() <= 1e-2 * want.norm()
    return got


@pytest.mark.parametrize("typ", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 50), (50, 1), (8, 8), (7, 13), (64, 64), (65, 63), (100, 333), (515, 129),
                                       (256, 1024), (600, 600)])
def test_update(ops, rows, cols, typ):
    grad = normal((rows, cols), typ, rows * 1000 + cols)
    check_update(ops, grad)
    check_update(ops, grad, momentum=normal((rows, cols), F32, 9, 3.0), dtype=F16)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("steps,coefficients", [(0, COEF), (1, COEF), (3, (1.5, -0.5, 0.0)),
                                                (2, ((2.0, -1.5, 0.5), (1.875, -1.25, 0.375)))])
def test_update_polynomials(ops, steps, coefficients, nesterov):
    grad = normal((40, 70), BF16, 4, 0.01)
    check_update(ops, grad, steps=steps, coefficients=coefficients, momentum=normal((40, 70), F32, 5), nesterov=nesterov)


@pytest.mark.parametrize("batch,rows,cols", [(3, 40, 24), (8, 128, 200), (2, 300, 310), (5, 1, 9)])
def test_update_batches(ops, batch, rows, cols):
    grad = normal((batch, rows, cols), F32, 6) * torch.tensor([10.0 ** -i for i in range(batch)], device="cuda").view(-1, 1, 1)
    check_update(ops, grad, momentum=torch.zeros_like(grad))


@pytest.mark.parametrize("rows,cols", [(1024, 2752), (2752, 1024)])
def test_update_larger(ops, rows, cols):
    check_update(ops, normal((rows, cols), BF16, 7))


@pytest.mark.parametrize("size", [1e-30, 1e-8, 1e8, 1e30])
def test_update_takes_any_magnitude(ops, size):
    """The squares of 1e30 pass float's range, those of 1e-30 fall below it."""
    grad = normal((60, 90), F32, 8)
    a = check_update(ops, grad * size, eps=0.0)
    b = check_update(ops, grad, eps=0.0)
    assert (a.double() - b.double()).norm() <= 1e-2 * b.double().norm()


def test_update_zero_and_bad_matrices(ops):
    grad = normal((4, 33, 20), BF16, 9)
    grad[1] = 0
    grad[2, 3, 4] = float("nan")
    for eps in (0.0, 1e-7):
        out = ops.orthogonal_update(grad, eps=eps)
        assert bool((out[1] == 0).all())
        assert torch.isnan(out[2]).any()
        assert torch.isfinite(out[0]).all() and torch.isfinite(out[3]).all()


def test_update_strides(ops):
    """Views with rows and matrices apart, starting on any value; outputs keep to theirs."""
    mem = normal((3, 50, 91), BF16, 10)
    grad = mem[:, 3:43, 5:82]
    box = torch.full((3, 44, 80), 7.0, dtype=BF16, device="cuda")
    out = box[:, 1:41, 1:78]
    mom = normal((3, 45, 83), F32, 11)
    keep = mom.clone()
    view = mom[:, 2:42, 3:80]
    want = ops.orthogonal_update(grad.contiguous(), momentum=view.contiguous())
    ops.orthogonal_update(grad, momentum=view, out=out)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((box == 7.0).all())
    view.copy_(keep[:, 2:42, 3:80])
    assert torch.equal(mom, keep)


# ---------------------------------------------------------------- streams, graphs, large offsets

def step(ops, t, weights, state, stream=None):
    """Forward, backward and update of a sub-layer; returns everything it writes."""
    wg, wu, wd = weights
    given = dict(gate=t["gate"], w_post=t["w_post"], scale=0.5, stream=stream)
    _, n, s0 = ops.norm_forward(t["x"], w_pre=t["w_pre"], dtype=BF16, save=True, stream=stream)
    y, saved = ops.ffn_forward(n, wg, wu, wd, save=True, stream=stream)
    r, _, s1 = ops.norm_forward(t["x"], y, next_norm=False, save=True, **given)
    b1 = ops.norm_backward(None, t["dr"], r, y, s1, **given)
    dn, *dw = ops.ffn_backward(b1["dy"], n, wg, wu, wd, saved, stream=stream)
    b0 = ops.norm_backward(dn, b1["dx"], t["x"], None, s0, w_pre=t["w_pre"], stream=stream)
    up = [ops.orthogonal_update(g, momentum=m, momentum_out=o, stream=stream) for g, (m, o) in zip(dw, state)]
    return [n, y, r, b0["dx"], b0["dw_pre"], b1["dgate"], b1["dw_post"], *dw, *up, *(o for _, o in state)]


def step_inputs(T=200, D=136, F=264):
    t = norm_inputs(T, D, BF16, F32, 0)
    _, wg, wu, wd, _ = ffn_inputs(1, D, F, BF16)
    state = [(normal(w.shape, F32, 20 + i), torch.empty(w.shape, device="cuda")) for i, w in enumerate((wg, wu, wd))]
    return t, (wg, wu, wd), state


def test_step_on_another_stream(ops):
    args = step_inputs()
    want = [v.clone() for v in step(ops, *args)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = step(ops, *args, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_step_is_captured_and_replayed(ops):
    args = step_inputs()
    want = [v.clone() for v in step(ops, *args)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(ops, *args)
    for _ in range(4):
        for v in out:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        again = step(ops, *args)       # eager work between replays
        assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_offsets_past_32_bits(ops):
    """Rows so far apart that element offsets pass 2^31 (and byte offsets 2^32)."""
    T, D, F, ld = 600, 64, 48, (1 << 22) - 8
    assert T * ld > 1 << 31
    x, wg, wu, wd, dy = ffn_inputs(T, D, F, BF16)
    far = torch.empty(T * ld, dtype=BF16, device="cuda").as_strided((T, D), (ld, 1))
    far.copy_(x)
    y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    assert torch.equal(ops.ffn_forward(far, wg, wu, wd), y)
    for a, b in zip(ops.ffn_backward(dy, far, wg, wu, wd, saved), ops.ffn_backward(dy, x, wg, wu, wd, saved)):
        assert torch.equal(a, b)
    assert torch.equal(ops.norm_forward(far)[1], ops.norm_forward(x)[1])


def test_refusals(ops):
    x, wg, wu, wd, dy = ffn_inputs(4, 32, 48, BF16)
    with pytest.raises(ValueError, match="activation"):
        ops.ffn_forward(x, wg, wu, wd, activation="tanh")
    with pytest.raises(ValueError, match="shape"):
        ops.ffn_forward(x, wg, wu[:-1], wd)
    with pytest.raises(ValueError, match="float16"):
        ops.ffn_forward(x, wg, wu, wd.half())
    with pytest.raises(ValueError, match="stride"):
        ops.ffn_forward(x.t().contiguous().t(), wg, wu, wd)
    with pytest.raises(ValueError, match="is on cpu"):
        ops.ffn_forward(x, wg.cpu(), wu, wd)
    with pytest.raises(arena.ArenaError, match="bfloat16 nor float16"):
        ops.ffn_forward(x.float(), wg.float(), wu.float(), wd.float())
    _, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    with pytest.raises(ValueError, match="saved"):
        ops.ffn_backward(dy[:2], x[:2], wg, wu, wd, saved)
    with pytest.raises(ValueError, match="accumulate"):
        ops.ffn_backward(dy, x, wg, wu, wd, saved, accumulate=True)
    with pytest.raises(ValueError, match="kind"):
        ops.norm_forward(x, kind="batch")
    with pytest.raises(ValueError, match="gate"):
        ops.norm_forward(x, dy, gate=torch.ones(2, 32, dtype=BF16, device="cuda"), gate_rows=1)
    with pytest.raises(ValueError, match="needs dn or dr"):
        ops.norm_backward(None, None, x, None, None)
    with pytest.raises(ValueError, match="two or three axes"):
        ops.orthogonal_update(x[0])
    with pytest.raises(ValueError, match="coefficients"):
        ops.orthogonal_update(x, coefficients=((1.5, -0.5, 0.0),) * 2, steps=3)
    with pytest.raises(ValueError, match="momentum"):
        ops.orthogonal_update(x, momentum=torch.zeros(4, 31, device="cuda"))
    with pytest.raises(arena.ArenaError, match="float16"):
        ops.orthogonal_update(x, coefficients=(17.0, 0.0, 0.0))


def test_rows_of_several_axes(ops):
    """[batch, tokens, model] tensors are their rows; rows that do not lie evenly are refused."""
    x, wg, wu, wd, _ = ffn_inputs(24, 32, 48, BF16)
    y = ops.ffn_forward(x, wg, wu, wd)
    assert torch.equal(ops.ffn_forward(x.view(4, 6, 32), wg, wu, wd), y.view(4, 6, 32))
    with pytest.raises(ValueError, match="evenly"):
        ops.ffn_forward(x.view(4, 6, 32)[:, :4], wg, wu, wd)
