"""The operators of a layer of experts and the cross entropy without a GPU: the headers'
functions are exported and bound, bad arguments are refused before any HIP call,
workspaces are sized, and the reference's formulas agree with differences."""
import ctypes
import os
import re
import subprocess
import types

import pytest
import torch

import experts_reference as exp
from paper_2403_16125_amd import arena, layer
from paper_2403_16125_amd import layer_experts as le

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000      # never dereferenced: validation reads pointers only
HEADERS = ("arena_experts.h", "arena_loss.h")


@pytest.fixture
def ctx():
    c = arena.arena_create(0)
    yield c
    arena.arena_destroy(c)


def test_header_functions_are_exported_and_bound():
    declared = set()
    for name in HEADERS:
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", name)).read(), flags=re.S)
        declared |= set(re.findall(r"\barena_status (arena_[a-z_]+)\s*\(", src))
    out = subprocess.run(["nm", "-D", "--defined-only", arena.library_path()], capture_output=True, text=True,
                         check=True).stdout
    assert declared == set(le.EXPORTED)
    assert declared <= set(re.findall(r"\bT (arena_[a-z_]+)", out))
    le.load()


@pytest.mark.parametrize("name,c", [("RouteDesc", "arena_route_desc"), ("SortDesc", "arena_sort_desc"),
                                    ("MoveDesc", "arena_move_desc"), ("ExpertsDesc", "arena_experts_desc"),
                                    ("ExpertsGrads", "arena_experts_grads"), ("LossDesc", "arena_loss_desc"),
                                    ("LossGrads", "arena_loss_grads")])
def test_descriptors_match_the_headers(name, c, tmp_path):
    cls = getattr(le, name)
    prints = "".join(f'printf("%zu ", offsetof({c}, {f}));' for f, _ in cls._fields_)
    src = tmp_path / "o.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "arena_loss.h"\n'
                   f'int main(void) {{ {prints} printf("%zu %d %d %d %d %d", sizeof({c}), ARENA_I32, ARENA_I64, '
                   f'ARENA_MAX_EXPERTS, ARENA_ROUTE_MAX_CHOICES, ARENA_MAX_CHOICES); return 0; }}\n')
    exe = str(tmp_path / "o")
    subprocess.run(["gcc", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(v) for v in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(cls, f).offset for f, _ in cls._fields_] + [
        ctypes.sizeof(cls), le.I32, le.I64, le.MAX_EXPERTS, le.ROUTE_MAX_CHOICES, le.MAX_CHOICES]


def refused(status, match, fn, *args):
    with pytest.raises(arena.ArenaError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)
    assert match in e.value.message, e.value.message


# ---------------------------------------------------------------- router

def route(**over):
    return le.RouteDesc(**{**dict(dtype=0, experts=8, k=2, normalise=1, tokens=4, scale=1.0, logits=FAKE, ld_logits=8,
                                  index=FAKE, weight=FAKE), **over})


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=3)), (1, "experts=0", dict(experts=0)), (5, "experts", dict(experts=1025, ld_logits=1025)),
    (1, "k=0", dict(k=0)), (5, "k=17", dict(k=17, experts=32, ld_logits=32)), (1, "of 8 experts", dict(k=9)),
    (1, "tokens", dict(tokens=-1)), (5, "tokens", dict(tokens=1 << 30)),
    (5, "choices", dict(tokens=(1 << 30) - 1, k=8)), (1, "scale", dict(scale=float("nan"))),
    (1, "logits is NULL", dict(logits=None)), (1, "less than its width", dict(ld_logits=7)),
    (1, "aligned", dict(logits=FAKE + 2)), (1, "index is NULL", dict(index=None)), (1, "weight is NULL", dict(weight=None)),
    (1, "aligned", dict(index=FAKE + 2)),
])
def test_route_refusals(ctx, status, match, over):
    refused(status, match, le.arena_route_forward, ctx, route(**over))


def test_route_backward_refusals(ctx):
    back = lambda d=None, dw=FAKE, ldw=2, dl=FAKE, ldl=8: le.arena_route_backward(ctx, d or route(), dw, ldw, dl, ldl)
    refused(1, "dweight is NULL", back, None, None)
    refused(1, "less than its width", back, None, FAKE, 1)
    refused(1, "dlogits is NULL", back, None, FAKE, 2, None)
    refused(1, "less than its width", back, None, FAKE, 2, FAKE, 7)
    refused(1, "index is NULL", back, route(index=None))
    refused(1, "descriptor is NULL", le.arena_route_backward, ctx, None, FAKE, 2, FAKE, 8)
    back(route(tokens=0, logits=None, index=None), None, 0, None, 0)


# ---------------------------------------------------------------- sort and moves

def sort(**over):
    return le.SortDesc(**{**dict(index_dtype=3, experts=8, tokens=4, k=2, index=FAKE, offsets=FAKE, row=FAKE), **over})


@pytest.mark.parametrize("status,match,over", [
    (1, "index_dtype", dict(index_dtype=0)), (1, "experts=0", dict(experts=0)), (5, "experts", dict(experts=1025)),
    (1, "k=0", dict(k=0)), (5, "k=65", dict(k=65)), (1, "tokens", dict(tokens=-1)), (5, "choices", dict(tokens=1 << 28, k=8)),
    (1, "index is NULL", dict(index=None)), (1, "offsets is NULL", dict(offsets=None)), (1, "row is NULL", dict(row=None)),
    (1, "aligned", dict(index=FAKE + 4, index_dtype=4)), (1, "workspace is NULL", dict(tokens=100000)),
])
def test_sort_refusals(ctx, status, match, over):
    refused(status, match, le.arena_sort_by_expert, ctx, sort(**over))


def test_sort_workspace(ctx):
    assert le.arena_sort_by_expert_workspace(ctx, sort()) == 0
    need = le.arena_sort_by_expert_workspace(ctx, sort(tokens=100000))
    assert 0 < need <= 128 * 8 * 4
    refused(1, "needed", le.arena_sort_by_expert, ctx, sort(tokens=100000, workspace=FAKE, workspace_bytes=need - 1))
    refused(1, "256 bytes", le.arena_sort_by_expert, ctx, sort(tokens=100000, workspace=FAKE + 8, workspace_bytes=need))


def move(**over):
    return le.MoveDesc(**{**dict(dtype=1, model=64, tokens=4, rows=8, k=2, row=FAKE, weight=FAKE, ld_weight=2), **over})


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=3)), (1, "model", dict(model=0)), (5, "model", dict(model=1 << 22)), (1, "k=0", dict(k=0)),
    (5, "k=65", dict(k=65)), (1, "tokens", dict(tokens=-1)), (1, "rows", dict(rows=-1)), (1, "row is NULL", dict(row=None)),
    (1, "weight is not aligned", dict(weight=FAKE + 2)),
])
def test_move_refusals(ctx, status, match, over):
    refused(status, match, le.arena_dispatch, ctx, move(**over), FAKE, 64, FAKE, 64)
    refused(status, match, le.arena_combine, ctx, move(**over), FAKE, 64, FAKE, 64)
    refused(status, match, le.arena_combine_backward, ctx, move(**over), FAKE, 64, FAKE, 64, FAKE, 64, FAKE)


def test_move_tensors_refused(ctx):
    for fn in (le.arena_dispatch, le.arena_combine):
        refused(1, "is NULL", fn, ctx, move(), None, 64, FAKE, 64)
        refused(1, "is NULL", fn, ctx, move(), FAKE, 64, None, 64)
        refused(1, "less than its width", fn, ctx, move(), FAKE, 63, FAKE, 64)
        refused(1, "aligned", fn, ctx, move(), FAKE, 64, FAKE + 1, 64)
        refused(5, "row stride", fn, ctx, move(), FAKE, 1 << 22, FAKE, 64)
    refused(1, "weight", le.arena_combine, ctx, move(ld_weight=1), FAKE, 64, FAKE, 64)
    back = lambda d, *a: le.arena_combine_backward(ctx, d, *a)
    refused(1, "weight is NULL", back, move(weight=None), FAKE, 64, FAKE, 64, FAKE, 64, FAKE)
    refused(1, "dweight is NULL", back, move(), FAKE, 64, FAKE, 64, FAKE, 64, None)
    refused(1, "dys is NULL", back, move(), FAKE, 64, FAKE, 64, None, 64, FAKE)


# ---------------------------------------------------------------- experts

def experts(**over):
    return le.ExpertsDesc(**{**dict(dtype=1, activation=0, rows=100, model=64, inner=96, experts=4, offsets=FAKE, x=FAKE, ld_x=64,
                                    w_gate=FAKE, ld_gate=64, stride_gate=6144, w_up=FAKE, ld_up=64, stride_up=6144, w_down=FAKE,
                                    ld_down=96, stride_down=6144, g=FAKE, u=FAKE, h=FAKE, ld_inner=96, y=FAKE, ld_y=64), **over})


def grads(**over):
    return le.ExpertsGrads(**{**dict(grad_dtype=1, accumulate=0, dy=FAKE, ld_dy=64, dx=FAKE, ld_dx=64, dw_gate=FAKE,
                                     ld_dw_gate=64, stride_dw_gate=6144, dw_up=FAKE, ld_dw_up=64, stride_dw_up=6144,
                                     dw_down=FAKE, ld_dw_down=96, stride_dw_down=6144), **over})


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=0)), (1, "activation", dict(activation=3)), (1, "rows", dict(rows=-1)), (1, "model", dict(model=0)),
    (1, "inner", dict(inner=0)), (5, "rows", dict(rows=1 << 30)), (5, "max", dict(model=1 << 22, ld_x=1 << 22)),
    (1, "experts=0", dict(experts=0)), (5, "experts", dict(experts=1025)), (1, "offsets is NULL", dict(offsets=None)),
    (1, "aligned", dict(offsets=FAKE + 2)), (1, "w_gate is NULL", dict(w_gate=None)), (1, "less than its width", dict(ld_down=95)),
    (1, "less than a matrix", dict(stride_up=6143)), (1, "less than a matrix", dict(stride_down=0)), (1, "x is NULL", dict(x=None)),
    (1, "y is NULL", dict(y=None)), (1, "h is NULL", dict(h=None)), (1, "together", dict(u=None)), (1, "16-byte", dict(h=FAKE + 2)),
    (1, "multiple of 8", dict(ld_inner=100)), (1, "aligned", dict(x=FAKE + 1)),
    (5, "too many tiles", dict(rows=(1 << 30) - 1, model=4000000, ld_x=4000000, ld_y=4000000, ld_gate=4000000, ld_up=4000000,
                               stride_gate=1 << 40, stride_up=1 << 40, stride_down=1 << 40)),
])
def test_experts_refusals(ctx, status, match, over):
    refused(status, match, le.arena_experts_forward, ctx, experts(**over))
    refused(status, match, le.arena_experts_forward_workspace, ctx, experts(**over))


def test_experts_strides_of_one_expert_do_not_matter(ctx):
    le.arena_experts_forward_workspace(ctx, experts(experts=1, stride_gate=0, stride_up=0, stride_down=0))


def test_experts_backward_refusals(ctx):
    size = lambda d, g: le.arena_experts_backward_workspace(ctx, d, g)
    need = size(experts(), grads())
    assert need >= 2 * 2 * 100 * 96
    refused(1, "needed", le.arena_experts_backward, ctx, experts(workspace=FAKE, workspace_bytes=need - 1), grads())
    refused(1, "workspace is NULL", le.arena_experts_backward, ctx, experts(), grads())
    for status, match, over in [(1, "grad_dtype", dict(grad_dtype=2)), (1, "dy is NULL", dict(dy=None)),
                                (1, "less than its width", dict(ld_dx=63)), (1, "less than a matrix", dict(stride_dw_gate=1)),
                                (1, "aligned", dict(dw_down=FAKE + 2, grad_dtype=0))]:
        refused(status, match, size, experts(), grads(**over))
    refused(1, "backward pass needs", size, experts(g=None, u=None), grads())
    refused(1, "descriptor is NULL", size, None, grads())
    refused(1, "descriptor is NULL", size, experts(), None)


# ---------------------------------------------------------------- cross entropy

def loss(**over):
    return le.LossDesc(**{**dict(dtype=1, target_dtype=4, tokens=100, model=64, vocabulary=1000, ignore_index=-100, x=FAKE,
                                 ld_x=64, w=FAKE, ld_w=64, target=FAKE, loss=FAKE, lse=FAKE), **over})


def loss_grads(**over):
    return le.LossGrads(**{**dict(grad_dtype=1, accumulate=0, dloss=FAKE, stride_dloss=1, dx=FAKE, ld_dx=64, dw=FAKE,
                                  ld_dw=64), **over})


@pytest.mark.parametrize("status,match,over", [
    (1, "dtype", dict(dtype=0)), (1, "target_dtype", dict(target_dtype=1)), (1, "tokens", dict(tokens=-1)),
    (1, "model", dict(model=0)), (1, "vocabulary", dict(vocabulary=0)), (5, "max", dict(vocabulary=(1 << 24) + 1)),
    (5, "max", dict(tokens=1 << 30)), (5, "max", dict(model=1 << 22)), (1, "x is NULL", dict(x=None)),
    (1, "w is NULL", dict(w=None)), (1, "target is NULL", dict(target=None)), (1, "lse is NULL", dict(lse=None)),
    (1, "less than its width", dict(ld_w=63)), (1, "aligned", dict(target=FAKE + 4)), (1, "aligned", dict(loss=FAKE + 2)),
    (5, "too many tiles", dict(tokens=(1 << 30) - 1, model=10000, ld_x=10000, ld_w=10000)),
])
def test_loss_refusals(ctx, status, match, over):
    refused(status, match, le.arena_cross_entropy_forward, ctx, loss(**over))
    refused(status, match, le.arena_cross_entropy_forward_workspace, ctx, loss(**over))
    refused(status, match, le.arena_cross_entropy_backward_workspace, ctx, loss(**over), loss_grads())


def test_loss_backward_refusals(ctx):
    size = lambda d, g: le.arena_cross_entropy_backward_workspace(ctx, d, g)
    need = size(loss(), loss_grads())
    refused(1, "needed", le.arena_cross_entropy_backward, ctx, loss(workspace=FAKE, workspace_bytes=need - 1), loss_grads())
    for status, match, over in [(1, "grad_dtype", dict(grad_dtype=2)), (1, "dloss is NULL", dict(dloss=None)),
                                (1, "stride_dloss", dict(stride_dloss=-1)), (1, "dloss is not aligned", dict(dloss=FAKE + 2)),
                                (1, "less than its width", dict(ld_dw=63)), (1, "less than its width", dict(ld_dx=63))]:
        refused(status, match, size, loss(), loss_grads(**over))
    refused(1, "descriptor is NULL", size, loss(), None)
    le.arena_cross_entropy_backward(ctx, loss(tokens=0), loss_grads(dw=None))


def test_loss_workspaces_are_bounded(ctx):
    """Neither direction's workspace grows with tokens times vocabulary past its pieces."""
    big = loss(tokens=65536, vocabulary=131072, model=4096, ld_x=4096, ld_w=4096)
    assert le.arena_cross_entropy_forward_workspace(ctx, big) <= 32768 * (131072 // 64 + 1) * 8
    g = loss_grads(ld_dx=4096, ld_dw=4096)
    rest = 65536 * 4096 * (2 + 4) + 65536 * 16       # x, the sum of dx, the tokens' records
    assert le.arena_cross_entropy_backward_workspace(ctx, big, g) <= rest + 65536 * 4096 * 2 + (1 << 28)


# ---------------------------------------------------------------- the binding's own checks

def test_binding_refuses_numbers_that_its_fields_would_cut_off():
    ops = layer.LayerOps()
    ops._current = lambda index: types.SimpleNamespace(cuda_stream=0)
    x, index = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for k in (0, -1, 2 ** 31, 2 ** 32 + 2):
        with pytest.raises(ValueError, match="k is"):
            ops.route(x, k)
        with pytest.raises(ValueError, match="experts is"):
            ops.sort_by_expert(index, k)
    for ignore in (2 ** 63, -2 ** 63 - 1, 2 ** 64):        # the last would be entry 0
        with pytest.raises(ValueError, match="ignore_index is"):
            ops.cross_entropy_forward(x.bfloat16(), x.bfloat16(), index[:, 0], ignore_index=ignore)
    ops.close()


def test_binding_refuses_what_is_not_on_the_device():
    ops = layer.LayerOps()
    ops._current = lambda index: types.SimpleNamespace(cuda_stream=0)      # no GPU is asked
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="logits is on cpu"):
        ops.route(x, 2)
    with pytest.raises(ValueError, match="index must be"):
        ops.sort_by_expert(torch.zeros(4, 2, dtype=torch.int32), 4)
    with pytest.raises(ValueError, match="not supported"):
        ops.route(x.double(), 2)
    with pytest.raises(ValueError, match="three axes"):
        ops.experts_forward(x.bfloat16(), torch.zeros(3, dtype=torch.int32), x, x, x)
    with pytest.raises(ValueError, match="requires a gradient"):
        ops.route(x.requires_grad_(), 2)
    ops.close()


# ---------------------------------------------------------------- formulas

@pytest.mark.parametrize("normalise", [True, False])
def test_route_gradient_of_the_reference(normalise):
    gen = torch.Generator().manual_seed(1)
    l = torch.randn(5, 7, generator=gen, dtype=torch.float64)
    l[1, 2:6] = -float("inf")
    index, weight = exp.route(l, 3, normalise, 1.5)
    dw = torch.randn(5, 3, generator=gen, dtype=torch.float64)
    f = lambda v: (exp.route_weight(v, index, normalise, 1.5) * dw).sum()
    assert torch.allclose(exp.route_weight(l, index, normalise, 1.5), weight, atol=1e-14)
    v, size = exp.route_back(dw, l, index, normalise, 1.5)
    for t in range(5):
        for e in range(7):
            if l[t, e] == -float("inf"):
                assert v[t, e] == 0
                continue
            h = torch.zeros_like(l)
            h[t, e] = 1e-6
            assert abs((f(l + h) - f(l - h)) / 2e-6 - v[t, e]) < 1e-8
    assert (v.abs() <= size + 1e-15).all()


def test_loss_gradient_of_the_reference():
    gen = torch.Generator().manual_seed(2)
    x, w = torch.randn(4, 3, generator=gen, dtype=torch.float64), torch.randn(6, 3, generator=gen, dtype=torch.float64)
    target, dloss = torch.tensor([1, -100, 5, 0]), torch.rand(4, generator=gen, dtype=torch.float64)
    f = lambda x, w: (exp.cross_entropy(x, w, target, -100, torch.bfloat16)["loss"][0] * dloss).sum()
    got = exp.cross_entropy(x, w, target, -100, torch.bfloat16, dloss)
    for name, at, other in (("dx", x, lambda d: f(x + d, w)), ("dw", w, lambda d: f(x, w + d))):
        for i in range(at.shape[0]):
            for j in range(3):
                d = torch.zeros_like(at)
                d[i, j] = 1e-6
                assert abs((other(d) - other(-d)) / 2e-6 - got[name][0][i, j]) < 1e-8
