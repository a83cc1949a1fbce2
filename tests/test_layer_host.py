"""The layer operators without a GPU: the header's functions are exported and
bound, bad arguments are refused before any HIP call, workspaces are sized, and
the reference's gradient formulas agree with differences of its definitions."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import layer_reference as ref
from paper_2403_16125_amd import arena, layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000      # never dereferenced: validation reads pointers only


@pytest.fixture
def ctx():
    c = arena.arena_create(0)
    yield c
    arena.arena_destroy(c)


def test_header_functions_are_exported_and_bound():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "arena_layer.h")).read(), flags=re.S)
    declared = set(re.findall(r"\barena_status (arena_[a-z_]+)\s*\(", src))
    out = subprocess.run(["nm", "-D", "--defined-only", arena.library_path()], capture_output=True, text=True,
                         check=True).stdout
    assert declared == set(layer.EXPORTED)
    assert declared <= set(re.findall(r"\bT (arena_[a-z_]+)", out))
    layer.load()


@pytest.mark.parametrize("name", ["NormDesc", "NormGrads", "FfnDesc", "FfnGrads", "UpdateDesc"])
def test_descriptors_match_the_header(name, tmp_path):
    """Sizes and offsets of the ctypes structures against a C compiler's."""
    c = {"NormDesc": "arena_norm_desc", "NormGrads": "arena_norm_grads", "FfnDesc": "arena_ffn_desc",
         "FfnGrads": "arena_ffn_grads", "UpdateDesc": "arena_update_desc"}[name]
    cls = getattr(layer, name)
    prints = "".join(f'printf("%zu ", offsetof({c}, {f}));' for f, _ in cls._fields_)
    src = tmp_path / "o.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "arena_layer.h"\n'
                   f'int main(void) {{ {prints} printf("%zu", sizeof({c})); return 0; }}\n')
    exe = str(tmp_path / "o")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(v) for v in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(cls, f).offset for f, _ in cls._fields_] + [ctypes.sizeof(cls)]


def _refused(status, match, fn, *args):
    with pytest.raises(arena.ArenaError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)
    assert match in e.value.message, e.value.message


def _norm(**over):
    d = dict(dtype=1, stream_dtype=0, kind=0, width=64, tokens=4, gate_rows=0, eps=1e-6, scale=1.0, x=FAKE, ld_x=64,
             y=FAKE, ld_y=64, r=FAKE, ld_r=64, n=FAKE, ld_n=64)
    d.update(over)
    return layer.NormDesc(**d)


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=3)), (1, "stream_dtype", dict(stream_dtype=2)), (1, "kind", dict(kind=2)),
    (1, "width", dict(width=0)), (5, "width", dict(width=16385, ld_x=16385)), (1, "tokens", dict(tokens=-1)),
    (5, "tokens", dict(tokens=1 << 30)), (1, "eps", dict(eps=float("nan"))), (1, "eps", dict(eps=-1.0)),
    (1, "scale", dict(scale=float("inf"))), (1, "need y", dict(y=None, gate=FAKE, ld_gate=64)),
    (1, "need n", dict(n=None, w_pre=FAKE)), (1, "nothing to do", dict(y=None, n=None)), (1, "x is NULL", dict(x=None)),
    (1, "r is NULL", dict(r=None)), (1, "less than its width", dict(ld_y=63)), (1, "aligned", dict(n=FAKE + 1)),
    (1, "aligned", dict(w_pre=FAKE + 1)), (5, "row stride", dict(ld_x=1 << 22)),
])
def test_norm_refusals(ctx, status, match, over):
    _refused(status, match, layer.arena_norm_forward, ctx, _norm(**over))


def test_norm_backward_refusals(ctx):
    f = _norm(stats=FAKE)
    g = lambda **o: layer.NormGrads(**{**dict(dn=FAKE, ld_dn=64, dx=FAKE, ld_dx=64), **o})
    run = lambda f, g: layer.arena_norm_backward(ctx, f, g)
    need = layer.arena_norm_backward_workspace(ctx, f)
    assert need > 0
    _refused(1, "workspace is NULL", run, f, g())
    _refused(1, "needed", run, f, g(workspace=FAKE, workspace_bytes=need - 1))
    _refused(1, "256 bytes", run, f, g(workspace=FAKE + 8, workspace_bytes=need))
    _refused(1, "neither dn nor dr", run, f, g(dn=None))
    _refused(1, "stats is NULL", run, _norm(), g())
    _refused(1, "dgate needs gate", run, f, g(dgate=FAKE))
    _refused(1, "need y", run, _norm(y=None, stats=FAKE), g(dy=FAKE, ld_dy=64))
    _refused(1, "descriptor is NULL", run, f, None)
    _refused(1, "descriptor is NULL", run, None, g())


def _ffn(**over):
    d = dict(dtype=1, activation=0, tokens=100, model=64, inner=96, x=FAKE, ld_x=64, w_gate=FAKE, ld_gate=64,
             w_up=FAKE, ld_up=64, w_down=FAKE, ld_down=96, g=FAKE, u=FAKE, h=FAKE, ld_inner=96, y=FAKE, ld_y=64)
    d.update(over)
    return layer.FfnDesc(**d)


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=0)), (1, "activation", dict(activation=3)), (1, "tokens", dict(tokens=-1)),
    (1, "model", dict(model=0)), (1, "inner", dict(inner=0)), (5, "tokens", dict(tokens=1 << 30)),
    (5, "max", dict(model=1 << 22, ld_x=1 << 22)), (1, "w_gate is NULL", dict(w_gate=None)),
    (1, "less than its width", dict(ld_down=95)), (1, "x is NULL", dict(x=None)), (1, "y is NULL", dict(y=None)),
    (1, "h is NULL", dict(h=None)), (1, "together", dict(u=None)), (1, "16-byte", dict(h=FAKE + 2)),
    (1, "16-byte", dict(g=FAKE + 8)), (1, "multiple of 8", dict(ld_inner=100)), (1, "less than", dict(inner=90, ld_inner=88)),
    (1, "aligned", dict(x=FAKE + 1)),
])
def test_ffn_refusals(ctx, status, match, over):
    _refused(status, match, layer.arena_ffn_forward, ctx, _ffn(**over))
    _refused(status, match, layer.arena_ffn_forward_workspace, ctx, _ffn(**over))


def test_ffn_backward_refusals(ctx):
    g = lambda **o: layer.FfnGrads(**{**dict(grad_dtype=1, accumulate=0, dy=FAKE, ld_dy=64, dx=FAKE, ld_dx=64,
                                             dw_gate=FAKE, ld_dw_gate=64, dw_up=FAKE, ld_dw_up=64, dw_down=FAKE,
                                             ld_dw_down=96), **o})
    run = lambda f, g: layer.arena_ffn_backward(ctx, f, g)
    assert layer.arena_ffn_backward_workspace(ctx, _ffn(), g()) >= 2 * 2 * 100 * 96
    _refused(1, "workspace is NULL", run, _ffn(), g())
    _refused(1, "backward pass needs them", run, _ffn(g=None, u=None), g())
    _refused(1, "grad_dtype", run, _ffn(), g(grad_dtype=2))
    _refused(1, "dy is NULL", run, _ffn(), g(dy=None))
    _refused(1, "less than its width", run, _ffn(), g(ld_dw_down=95))
    _refused(1, "aligned", run, _ffn(), g(grad_dtype=0, dw_up=FAKE + 2))
    _refused(1, "descriptor is NULL", run, _ffn(), None)


def test_ffn_workspace_counts_copies_and_splits(ctx):
    # everything in place and wide enough not to be split: nothing
    big = dict(tokens=8192, model=4096, inner=8192, ld_x=4096, ld_gate=4096, ld_up=4096, ld_down=8192, ld_inner=8192, ld_y=4096)
    assert layer.arena_ffn_forward_workspace(ctx, _ffn(**big)) == 0
    # few tokens read unaligned operands in place
    assert layer.arena_ffn_forward_workspace(ctx, _ffn(tokens=1, x=FAKE + 2, w_gate=FAKE + 2, w_up=FAKE + 2)) == 0
    # an odd stride means a copy with rows of multiples of 8
    assert layer.arena_ffn_forward_workspace(ctx, _ffn(**{**big, "ld_x": 4097})) == 2 * 8192 * 4096
    assert layer.arena_ffn_forward_workspace(ctx, _ffn(tokens=0)) == 0


COEF = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)


def _update(**over):
    d = dict(dtype=0, out_dtype=1, batch=1, rows=32, cols=48, steps=1, nesterov=1, mu=0.95, eps=1e-7, scale=1.0,
             coefficients=ctypes.addressof(COEF), grad=FAKE, ld_grad=48, out=FAKE, ld_out=48)
    d.update(over)
    return layer.UpdateDesc(**d)


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=5)), (1, "out_dtype", dict(out_dtype=0)), (1, "rows", dict(rows=0)),
    (1, "batch", dict(batch=0)), (1, "steps", dict(steps=-1)), (5, "max", dict(rows=32769)), (5, "max", dict(steps=17)),
    (5, "max", dict(batch=4097)), (1, "finite", dict(mu=float("nan"))), (1, "eps", dict(eps=-1.0)),
    (1, "coefficients is NULL", dict(coefficients=None)), (1, "together", dict(momentum=FAKE, ld_momentum=48)),
    (1, "grad is NULL", dict(grad=None)), (1, "less than its width", dict(ld_out=47)), (1, "aligned", dict(grad=FAKE + 2)),
    (1, "less than a matrix", dict(batch=2, stride_grad=32 * 48 - 1, stride_out=32 * 48)),
])
def test_update_refusals(ctx, status, match, over):
    _refused(status, match, layer.arena_orthogonal_update, ctx, _update(**over))
    _refused(status, match, layer.arena_orthogonal_update_workspace, ctx, _update(**over))


@pytest.mark.parametrize("coefficients,ok", [
    ((1.5, -0.5, 0.0), True), ((2.0, -1.5, 0.5), True), ((3.4445, -4.7750, 2.0315), True), ((0.0, 0.0, 0.0), True),
    ((16.0, 0.0, 0.0), False), ((1.0, 20.0, 0.0), False), ((1.0, 0.0, 40.0), False), ((3.95, 0.0, 0.0), False),
])
def test_polynomials_that_leave_float16_are_refused(ctx, coefficients, ok):
    """Two steps of each: (3.95, 0, 0) takes a singular value of 1 to 3.95, whose square passes the limit."""
    table = (ctypes.c_float * 6)(*(coefficients * 2))
    d = _update(steps=2, coefficients=ctypes.addressof(table))
    if ok:
        assert layer.arena_orthogonal_update_workspace(ctx, d) > 0
    else:
        _refused(5, "float16", layer.arena_orthogonal_update_workspace, ctx, d)
    table[0] = float("inf")
    _refused(1, "not finite", layer.arena_orthogonal_update_workspace, ctx, d)


def test_null_context():
    lib = layer.load()
    assert lib.arena_norm_forward(None, None, None) == 1
    assert lib.arena_ffn_forward(None, None, None) == 1
    assert lib.arena_orthogonal_update(None, None, None) == 1


# ---------------------------------------------------------------- the reference itself

def _difference(f, t, at, h=1e-5):
    v = t.view(-1)
    keep = v[at].item()
    v[at] = keep + h
    hi = f()
    v[at] = keep - h
    lo = f()
    v[at] = keep
    return (hi - lo) / (2 * h)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_ffn_formulas_against_differences(name):
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    t = dict(x=r(3, 5), wg=r(7, 5), wu=r(7, 5), wd=r(5, 7))
    dy = r(3, 5)
    _, _, kept = ref.ffn(t["x"], t["wg"], t["wu"], t["wd"], name, torch.float32)
    got = ref.ffn_back(dy, t["x"], t["wg"], t["wu"], t["wd"], name, torch.float32, kept)
    f = lambda: (ref.ffn(t["x"], t["wg"], t["wu"], t["wd"], name, torch.float32)[0] * dy).sum().item()
    for key, grad in (("x", "dx"), ("wg", "dw_gate"), ("wu", "dw_up"), ("wd", "dw_down")):
        for at in range(0, t[key].numel(), 3):
            want = _difference(f, t[key], at)
            assert abs(got[grad][0].reshape(-1)[at].item() - want) <= 1e-6 * (1 + abs(want)), (grad, at)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows", [0, 1, 2, 4])
def test_norm_formulas_against_differences(kind, rows):
    gen = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    T, D, eps, scale = 5, 6, 1e-3, 0.7
    groups = -(-T // rows) if rows else 1
    t = dict(x=r(T, D), y=r(T, D), gate=r(groups, D), w_post=r(D), b_post=r(D), w_pre=r(D), b_pre=r(D))
    dn, dr = r(T, D), r(T, D)

    def both():
        return ref.block(t["x"], t["y"], t["gate"], rows, scale, t["w_post"], t["b_post"], t["w_pre"], t["b_pre"],
                         kind, eps)

    res, _ = both()
    _, m2, s2 = ref.norm(t["y"], kind, eps)
    _, m1, s1 = ref.norm(res, kind, eps)
    got = ref.block_back(dn, dr, res, t["y"], torch.cat([m2, s2, m1, s1], 1), t["gate"], rows, scale, t["w_post"],
                         t["b_post"], t["w_pre"], kind)

    def f():
        a, b = both()
        return ((a * dr).sum() + (b * dn).sum()).item()

    for key in t:
        for at in range(0, t[key].numel(), 2):
            want = _difference(f, t[key], at)
            assert abs(got["d" + key].reshape(-1)[at].item() - want) <= 1e-5 * (1 + abs(want)), (key, at)
