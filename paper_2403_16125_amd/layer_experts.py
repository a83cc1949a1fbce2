"""Python binding of the operators of a mixture-of-experts layer and of the
vocabulary's cross entropy (include/arena_experts.h, include/arena_loss.h), as
methods of layer.LayerOps.

The raw functions carry the C ABI's names.  `ExpertOps` checks shapes and types,
makes outputs and workspaces, and enqueues on the current stream (or the one
given), as the other operators of LayerOps do.
"""
from __future__ import annotations

import ctypes
import dataclasses

from . import arena
from .arena import _check

I32, I64 = 3, 4
MAX_EXPERTS, ROUTE_MAX_CHOICES, MAX_CHOICES = 1024, 16, 64
IGNORE_INDEX = -100

EXPORTED = (
    "arena_route_forward", "arena_route_backward", "arena_sort_by_expert_workspace", "arena_sort_by_expert",
    "arena_dispatch", "arena_combine", "arena_combine_backward", "arena_experts_forward_workspace",
    "arena_experts_forward", "arena_experts_backward_workspace", "arena_experts_backward",
    "arena_cross_entropy_forward_workspace", "arena_cross_entropy_forward", "arena_cross_entropy_backward_workspace",
    "arena_cross_entropy_backward",
)

_i32, _i64, _f32, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class RouteDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("experts", _i32), ("k", _i32), ("normalise", _i32), ("tokens", _i64),
                ("scale", _f32), ("logits", _vp), ("ld_logits", _i64), ("index", _vp), ("weight", _vp)]


class SortDesc(ctypes.Structure):
    _fields_ = [("index_dtype", _i32), ("experts", _i32), ("tokens", _i64), ("k", _i32), ("index", _vp),
                ("offsets", _vp), ("row", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class MoveDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("model", _i32), ("tokens", _i64), ("rows", _i64), ("k", _i32), ("row", _vp),
                ("weight", _vp), ("ld_weight", _i64)]


class ExpertsDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("activation", _i32), ("rows", _i64), ("model", _i32), ("inner", _i32),
                ("experts", _i32), ("offsets", _vp), ("x", _vp), ("ld_x", _i64), ("w_gate", _vp), ("ld_gate", _i64),
                ("stride_gate", _i64), ("w_up", _vp), ("ld_up", _i64), ("stride_up", _i64), ("w_down", _vp),
                ("ld_down", _i64), ("stride_down", _i64), ("g", _vp), ("u", _vp), ("h", _vp), ("ld_inner", _i64),
                ("y", _vp), ("ld_y", _i64), ("workspace", _vp), ("workspace_bytes", _i64)]


class ExpertsGrads(ctypes.Structure):
    _fields_ = [("grad_dtype", _i32), ("accumulate", _i32), ("dy", _vp), ("ld_dy", _i64), ("dx", _vp),
                ("ld_dx", _i64), ("dw_gate", _vp), ("ld_dw_gate", _i64), ("stride_dw_gate", _i64), ("dw_up", _vp),
                ("ld_dw_up", _i64), ("stride_dw_up", _i64), ("dw_down", _vp), ("ld_dw_down", _i64),
                ("stride_dw_down", _i64)]


class LossDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("target_dtype", _i32), ("tokens", _i64), ("model", _i32), ("vocabulary", _i32),
                ("ignore_index", _i64), ("x", _vp), ("ld_x", _i64), ("w", _vp), ("ld_w", _i64), ("target", _vp),
                ("loss", _vp), ("lse", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class LossGrads(ctypes.Structure):
    _fields_ = [("grad_dtype", _i32), ("accumulate", _i32), ("dloss", _vp), ("stride_dloss", _i64), ("dx", _vp),
                ("ld_dx", _i64), ("dw", _vp), ("ld_dw", _i64)]


_bound = None


def load():
    """The library with these operators' signatures; raises if it has not been built."""
    global _bound
    lib = arena._lib
    if lib is not None and _bound is lib:
        return lib
    lib = arena.load()
    P, out = ctypes.POINTER, ctypes.POINTER(_i64)
    signatures = {
        "arena_route_forward": [_vp, P(RouteDesc), _vp],
        "arena_route_backward": [_vp, P(RouteDesc), _vp, _i64, _vp, _i64, _vp],
        "arena_sort_by_expert_workspace": [_vp, P(SortDesc), out],
        "arena_sort_by_expert": [_vp, P(SortDesc), _vp],
        "arena_dispatch": [_vp, P(MoveDesc), _vp, _i64, _vp, _i64, _vp],
        "arena_combine": [_vp, P(MoveDesc), _vp, _i64, _vp, _i64, _vp],
        "arena_combine_backward": [_vp, P(MoveDesc), _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp],
        "arena_experts_forward_workspace": [_vp, P(ExpertsDesc), out],
        "arena_experts_forward": [_vp, P(ExpertsDesc), _vp],
        "arena_experts_backward_workspace": [_vp, P(ExpertsDesc), P(ExpertsGrads), out],
        "arena_experts_backward": [_vp, P(ExpertsDesc), P(ExpertsGrads), _vp],
        "arena_cross_entropy_forward_workspace": [_vp, P(LossDesc), out],
        "arena_cross_entropy_forward": [_vp, P(LossDesc), _vp],
        "arena_cross_entropy_backward_workspace": [_vp, P(LossDesc), P(LossGrads), out],
        "arena_cross_entropy_backward": [_vp, P(LossDesc), P(LossGrads), _vp],
    }
    for name, args in signatures.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    _bound = lib
    return lib


# ---------------------------------------------------------------- raw C ABI

def _ref(d):
    return None if d is None else ctypes.byref(d)


def arena_route_forward(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_route_forward(ctx, _ref(desc), stream))


def arena_route_backward(ctx, desc, dweight, ld_dweight, dlogits, ld_dlogits, stream=0) -> None:
    _check(ctx, load().arena_route_backward(ctx, _ref(desc), dweight, ld_dweight, dlogits, ld_dlogits, stream))


def arena_sort_by_expert_workspace(ctx, desc) -> int:
    n = _i64()
    _check(ctx, load().arena_sort_by_expert_workspace(ctx, _ref(desc), ctypes.byref(n)))
    return n.value


def arena_sort_by_expert(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_sort_by_expert(ctx, _ref(desc), stream))


def arena_dispatch(ctx, desc, x, ld_x, xs, ld_xs, stream=0) -> None:
    _check(ctx, load().arena_dispatch(ctx, _ref(desc), x, ld_x, xs, ld_xs, stream))


def arena_combine(ctx, desc, ys, ld_ys, y, ld_y, stream=0) -> None:
    _check(ctx, load().arena_combine(ctx, _ref(desc), ys, ld_ys, y, ld_y, stream))


def arena_combine_backward(ctx, desc, dy, ld_dy, ys, ld_ys, dys, ld_dys, dweight, stream=0) -> None:
    _check(ctx, load().arena_combine_backward(ctx, _ref(desc), dy, ld_dy, ys, ld_ys, dys, ld_dys, dweight, stream))


def arena_experts_forward_workspace(ctx, desc) -> int:
    n = _i64()
    _check(ctx, load().arena_experts_forward_workspace(ctx, _ref(desc), ctypes.byref(n)))
    return n.value


def arena_experts_forward(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_experts_forward(ctx, _ref(desc), stream))


def arena_experts_backward_workspace(ctx, desc, grads) -> int:
    n = _i64()
    _check(ctx, load().arena_experts_backward_workspace(ctx, _ref(desc), _ref(grads), ctypes.byref(n)))
    return n.value


def arena_experts_backward(ctx, desc, grads, stream=0) -> None:
    _check(ctx, load().arena_experts_backward(ctx, _ref(desc), _ref(grads), stream))


def arena_cross_entropy_forward_workspace(ctx, desc) -> int:
    n = _i64()
    _check(ctx, load().arena_cross_entropy_forward_workspace(ctx, _ref(desc), ctypes.byref(n)))
    return n.value


def arena_cross_entropy_forward(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_cross_entropy_forward(ctx, _ref(desc), stream))


def arena_cross_entropy_backward_workspace(ctx, desc, grads) -> int:
    n = _i64()
    _check(ctx, load().arena_cross_entropy_backward_workspace(ctx, _ref(desc), _ref(grads), ctypes.byref(n)))
    return n.value


def arena_cross_entropy_backward(ctx, desc, grads, stream=0) -> None:
    _check(ctx, load().arena_cross_entropy_backward(ctx, _ref(desc), _ref(grads), stream))


# ---------------------------------------------------------------- torch tensors

@dataclasses.dataclass
class ExpertPlan:
    """Tokens sorted by expert: rows offsets[e] .. offsets[e + 1] - 1 are expert e's,
    row[..., j] is that of a token's choice j, -1 where it is dropped (int32, on the
    device).  There is room for every choice: rows past offsets[-1] are no one's."""
    offsets: object
    row: object

    @property
    def rows(self) -> int:
        return self.row.numel()


class ExpertOps:
    """The methods of LayerOps for layers of experts and for the loss."""

    # -- checks

    @staticmethod
    def _within(name, value, bits, least=1):
        """A number that the descriptors' fields would cut off is refused."""
        if not least <= value < 1 << (bits - 1):
            raise ValueError(f"{name} is {value}")

    def _choices(self, name, t):
        """Tokens, and choices of a token, of a tensor with a value a choice."""
        if t.dim() < 1:
            raise ValueError(f"{name} needs an axis of choices")
        tokens, k = self._rows(t)
        if k >> 31:
            raise ValueError(f"{name} has {k} choices a token")
        return tokens, k

    def _whole(self, name, t, shape):
        """Address and type of a contiguous tensor of int32 or int64."""
        wide = t.dtype is self.torch.int64
        if t.get_device() != self._index or not (wide or t.dtype is self.torch.int32) or t.shape != shape \
                or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 or int64 tensor of shape {tuple(shape)} on {self.dev}")
        return t.data_ptr(), I64 if wide else I32

    def _int32(self, name, t, shape):
        p, kind = self._whole(name, t, shape)
        if kind != I32:
            raise ValueError(f"{name} is {t.dtype}, not int32")
        return p

    def _float32(self, name, t, shape):
        if t.get_device() != self._index or t.dtype is not self.torch.float32 or t.shape != shape \
                or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 tensor of shape {tuple(shape)} on {self.dev}")
        return t.data_ptr()

    def _output(self, name, out, shape, dtype):
        """An output, new unless given, as a matrix: tensor, address and row stride."""
        if out is None:
            out = self._empty(shape, dtype)
        p, ld = self._matrix(name, out, self._rows(out), dtype)
        if out.shape != shape:
            raise ValueError(f"{name} has shape {tuple(out.shape)}, not {tuple(shape)}")
        return out, p, ld

    # -- router

    def route(self, logits, k, *, normalise=True, scale=1.0, stream=None):
        """(index, weight) of each token's k experts: the k largest of logits
        [..., experts] in falling order, of equal ones the lowest index first (int32
        [..., k]), and scale times their softmax, over the chosen (normalise) or over
        all (float32 [..., k]).  An expert whose logit is -inf is never chosen:
        choices that are left over have index -1 and weight 0."""
        return self._run(stream, (logits,), self._route, logits, k, normalise, scale)

    def _route_desc(self, logits, k, normalise, scale):
        tokens, experts = self._rows(logits)
        d = RouteDesc(dtype=self._type(logits), experts=experts, k=k, normalise=int(bool(normalise)), tokens=tokens,
                      scale=scale)
        d.logits, d.ld_logits = self._matrix("logits", logits, (tokens, experts), logits.dtype)
        return d

    def _route(self, handle, logits, k, normalise, scale):
        self._within("k", k, 32)
        d = self._route_desc(logits, k, normalise, scale)
        shape = logits.shape[:-1] + (k,)
        index, weight = self._empty(shape, self.torch.int32), self._empty(shape, self.torch.float32)
        d.index, d.weight = index.data_ptr(), weight.data_ptr()
        arena_route_forward(self.ctx, d, handle)
        return index, weight

    def route_backward(self, dweight, logits, index, *, normalise=True, scale=1.0, stream=None):
        """dlogits from the weights' gradient (float32 [..., k]), with the logits and
        the index of the forward pass."""
        return self._run(stream, (dweight, logits, index), self._route_backward, dweight, logits, index, normalise, scale)

    def _route_backward(self, handle, dweight, logits, index, normalise, scale):
        k = self._choices("index", index)[1]
        d = self._route_desc(logits, k, normalise, scale)
        d.index = self._int32("index", index, logits.shape[:-1] + (k,))
        p, ld = self._matrix("dweight", dweight, (d.tokens, k), self.torch.float32)
        dlogits = self._empty(logits.shape, logits.dtype)
        arena_route_backward(self.ctx, d, p, ld, dlogits.data_ptr(), d.experts, handle)
        return dlogits

    # -- tokens to experts and back

    def sort_by_expert(self, index, experts, *, stream=None):
        """The ExpertPlan of choices index [..., k] (int32 or int64): rows in order
        of their expert, within one in order of the tokens and their choices.  An index
        outside of 0..experts-1 (route's -1) is a dropped choice."""
        return self._run(stream, (index,), self._sort_by_expert, index, experts)

    def _sort_by_expert(self, handle, index, experts):
        self._within("experts", experts, 32)
        tokens, k = self._choices("index", index)
        p, kind = self._whole("index", index, index.shape)
        plan = ExpertPlan(self._empty((experts + 1,), self.torch.int32), self._empty(index.shape, self.torch.int32))
        d = SortDesc(index_dtype=kind, experts=experts, tokens=tokens, k=k, index=p, offsets=plan.offsets.data_ptr(),
                     row=plan.row.data_ptr())
        keep = self._workspace(d, arena_sort_by_expert_workspace(self.ctx, d))
        arena_sort_by_expert(self.ctx, d, handle)
        del keep
        return plan

    def _move_desc(self, dtype, model, plan, rows, weight=None):
        row = plan.row
        tokens, k = self._choices("plan.row", row)
        d = MoveDesc(dtype=self._code(dtype), model=model, tokens=tokens, rows=rows, k=k,
                     row=self._int32("plan.row", row, row.shape))
        if weight is not None:
            d.weight, d.ld_weight = self._matrix("weight", weight, (tokens, k), self.torch.float32)
        return d

    def dispatch(self, x, plan, *, out=None, stream=None):
        """xs [plan.rows, model] from x [..., model], each token's row copied to those of
        its choices.  Rows past plan.offsets[-1] are not written."""
        return self._run(stream, (x, plan.row, out), self._dispatch, x, plan, out)

    def _dispatch(self, handle, x, plan, out):
        model = x.shape[-1]
        xs, q, ld_q = self._output("out", out, (plan.rows, model), x.dtype)
        d = self._move_desc(x.dtype, model, plan, plan.rows)
        p, ld_p = self._matrix("x", x, (d.tokens, model), x.dtype)
        arena_dispatch(self.ctx, d, p, ld_p, q, ld_q, handle)
        return xs

    def combine(self, ys, plan, weight=None, *, out=None, stream=None):
        """y [..., model], the sum of each token's rows of ys [rows, model], each times
        its weight (float32 [..., k]; None: 1), over the choices that are not dropped."""
        return self._run(stream, (ys, plan.row, weight, out), self._combine, ys, plan, weight, out)

    def _combine(self, handle, ys, plan, weight, out):
        rows, model = self._rows(ys)
        d = self._move_desc(ys.dtype, model, plan, rows, weight)
        y, q, ld_q = self._output("out", out, plan.row.shape[:-1] + (model,), ys.dtype)
        p, ld_p = self._matrix("ys", ys, (rows, model), ys.dtype)
        arena_combine(self.ctx, d, p, ld_p, q, ld_q, handle)
        return y

    def combine_backward(self, dy, ys, plan, weight, *, out=None, stream=None):
        """(dys, dweight) from dy, the gradient of combine's y.  Rows of dys (new, or
        `out`) that no choice names are not written."""
        return self._run(stream, (dy, ys, plan.row, weight, out), self._combine_backward, dy, ys, plan, weight, out)

    def _combine_backward(self, handle, dy, ys, plan, weight, out):
        rows, model = self._rows(ys)
        d = self._move_desc(ys.dtype, model, plan, rows, weight)
        dys, r, ld_r = self._output("out", out, (rows, model), ys.dtype)
        dweight = self._empty(plan.row.shape, self.torch.float32)
        p, ld_p = self._matrix("dy", dy, (d.tokens, model), ys.dtype)
        q, ld_q = self._matrix("ys", ys, (rows, model), ys.dtype)
        arena_combine_backward(self.ctx, d, p, ld_p, q, ld_q, r, ld_r, dweight.data_ptr(), handle)
        return dys, dweight

    def dispatch_backward(self, dxs, plan, *, out=None, stream=None):
        """dx from dxs, the gradient of dispatch's xs: the sum over a token's choices."""
        return self.combine(dxs, plan, out=out, stream=stream)

    # -- experts' gated blocks

    def _experts_desc(self, xs, offsets, w_gate, w_up, w_down, activation):
        rows, model = self._rows(xs)
        if w_gate.dim() != 3:
            raise ValueError("the weights have three axes: experts, rows and columns")
        experts, inner = w_gate.shape[:2]
        if experts >> 31:
            raise ValueError(f"w_gate has {experts} experts")
        d = ExpertsDesc(dtype=self._type(xs), activation=self._activation(activation), rows=rows, model=model, inner=inner,
                        experts=experts, offsets=self._int32("offsets", offsets, (experts + 1,)))
        d.x, d.ld_x = self._matrix("xs", xs, (rows, model), xs.dtype)
        d.w_gate, d.ld_gate, d.stride_gate = self._stack("w_gate", w_gate, (experts, inner, model), xs.dtype)
        d.w_up, d.ld_up, d.stride_up = self._stack("w_up", w_up, (experts, inner, model), xs.dtype)
        d.w_down, d.ld_down, d.stride_down = self._stack("w_down", w_down, (experts, model, inner), xs.dtype)
        return d

    def experts_forward(self, xs, offsets, w_gate, w_up, w_down, *, activation="silu", save=False, out=None,
                        stream=None):
        """ys: rows offsets[e] .. offsets[e + 1] - 1 of xs [rows, model] through expert
        e's gated block (ffn_forward's), with w_gate and w_up [experts, inner, model]
        and w_down [experts, model, inner].  offsets: int32 [experts + 1] on the device,
        not falling, as an ExpertPlan's.  Rows outside of all groups are neither read
        nor written.  Returns ys, with save=True (ys, FfnSaved) for experts_backward."""
        return self._run(stream, (xs, offsets, w_gate, w_up, w_down, out), self._experts_forward, xs, offsets, w_gate,
                         w_up, w_down, activation, save, out)

    def _experts_forward(self, handle, xs, offsets, w_gate, w_up, w_down, activation, save, out):
        d = self._experts_desc(xs, offsets, w_gate, w_up, w_down, activation)
        ys, d.y, d.ld_y = self._output("out", out, xs.shape, xs.dtype)
        saved, base, g, u = self._inner(d.rows, d.inner, save)
        d.h, d.ld_inner = base, saved.ld
        if save:
            d.g, d.u = base + g, base + u
        keep = self._workspace(d, arena_experts_forward_workspace(self.ctx, d))
        arena_experts_forward(self.ctx, d, handle)
        del keep
        return (ys, saved) if save else ys

    def experts_backward(self, dys, xs, offsets, w_gate, w_up, w_down, saved, *, activation="silu", grads=None,
                         accumulate=False, stream=None):
        """(dxs, dw_gate, dw_up, dw_down) from dys, with the forward's inputs and
        `saved`.  Rows of dxs outside of all groups are not written; the weights'
        gradients of an expert without rows are zero.  grads: three tensors for the
        weights' gradients, of xs's type or float32, which accumulate=True adds to."""
        return self._run(stream, (dys, xs, offsets, w_gate, w_up, w_down, saved.buffer, *(() if grads is None else grads)),
                         self._experts_backward, dys, xs, offsets, w_gate, w_up, w_down, saved, activation, grads,
                         accumulate)

    def _experts_backward(self, handle, dys, xs, offsets, w_gate, w_up, w_down, saved, activation, grads, accumulate):
        d = self._experts_desc(xs, offsets, w_gate, w_up, w_down, activation)
        if accumulate and grads is None:
            raise ValueError("accumulate needs the gradients to add to")
        d.ld_inner = -(-d.inner // 8) * 8
        _, at_g, at_u, size = saved.parts()
        if (saved.tokens, saved.ld) != (d.rows, d.ld_inner) or saved.buffer.numel() != size \
                or saved.buffer.device != self.dev:
            raise ValueError("saved is not what experts_forward returned for these inputs")
        base = saved.buffer.data_ptr()
        d.h, d.g, d.u = base, base + at_g, base + at_u
        g = ExpertsGrads(accumulate=int(bool(accumulate)))
        g.dy, g.ld_dy = self._matrix("dys", dys, (d.rows, d.model), xs.dtype)
        dxs = self._empty(xs.shape, xs.dtype)
        g.dx, g.ld_dx = dxs.data_ptr(), d.model
        if grads is None:
            grads = tuple(self._empty(w.shape, xs.dtype) for w in (w_gate, w_up, w_down))
        kind = grads[0].dtype
        g.grad_dtype = self._type(grads[0])
        g.dw_gate, g.ld_dw_gate, g.stride_dw_gate = self._stack("dw_gate", grads[0], w_gate.shape, kind)
        g.dw_up, g.ld_dw_up, g.stride_dw_up = self._stack("dw_up", grads[1], w_up.shape, kind)
        g.dw_down, g.ld_dw_down, g.stride_dw_down = self._stack("dw_down", grads[2], w_down.shape, kind)
        keep = self._workspace(d, arena_experts_backward_workspace(self.ctx, d, g))
        arena_experts_backward(self.ctx, d, g, handle)
        del keep
        return (dxs, *grads)

    # -- cross entropy over a vocabulary

    def _loss_desc(self, x, w, target, ignore_index):
        self._within("ignore_index", ignore_index, 64, -1 << 63)
        tokens, model = self._rows(x)
        d = LossDesc(dtype=self._type(x), tokens=tokens, model=model, vocabulary=w.shape[0], ignore_index=ignore_index)
        d.x, d.ld_x = self._matrix("x", x, (tokens, model), x.dtype)
        d.w, d.ld_w = self._matrix("w", w, (d.vocabulary, model), x.dtype)
        d.target, d.target_dtype = self._whole("target", target, x.shape[:-1])
        return d

    def cross_entropy_forward(self, x, w, target, *, ignore_index=IGNORE_INDEX, stream=None):
        """(loss, lse) of each token: lse the log of the sum of the exponentials of its
        logits x w^T, loss lse less the target's logit, float32 [...].  x: [...,
        model], w: [vocabulary, model], bfloat16 or float16; target: int32 or int64 [...].
        The logits are not kept.  The loss is 0 where the target is ignore_index, NaN where
        it is any other value that is no entry of the vocabulary."""
        return self._run(stream, (x, w, target), self._cross_entropy_forward, x, w, target, ignore_index)

    def _cross_entropy_forward(self, handle, x, w, target, ignore_index):
        d = self._loss_desc(x, w, target, ignore_index)
        loss, lse = (self._empty(target.shape, self.torch.float32) for _ in range(2))
        d.loss, d.lse = loss.data_ptr(), lse.data_ptr()
        keep = self._workspace(d, arena_cross_entropy_forward_workspace(self.ctx, d))
        arena_cross_entropy_forward(self.ctx, d, handle)
        del keep
        return loss, lse

    def cross_entropy_backward(self, dloss, x, w, target, lse, *, ignore_index=IGNORE_INDEX, dw=None, accumulate=False,
                               stream=None):
        """(dx, dw) from dloss, the losses' gradient (float32 [...], or one value for
        all tokens), with the forward's inputs and lse.  dw: a tensor for the weight's
        gradient, of x's type or float32, which accumulate=True adds to."""
        return self._run(stream, (dloss, x, w, target, lse, dw), self._cross_entropy_backward, dloss, x, w, target, lse,
                         ignore_index, dw, accumulate)

    def _cross_entropy_backward(self, handle, dloss, x, w, target, lse, ignore_index, dw, accumulate):
        d = self._loss_desc(x, w, target, ignore_index)
        if accumulate and dw is None:
            raise ValueError("accumulate needs the gradient to add to")
        d.lse = self._float32("lse", lse, target.shape)
        g = LossGrads(accumulate=int(bool(accumulate)))
        if dloss.get_device() != self._index or dloss.dtype is not self.torch.float32 or \
                (dloss.dim() and dloss.shape != target.shape):
            raise ValueError(f"dloss must be float32 of shape {tuple(target.shape)}, or one value, on {self.dev}")
        if any(dloss.stride()):
            try:
                g.stride_dloss = dloss.view(-1).stride(0)
            except RuntimeError:
                raise ValueError(f"dloss: values of shape {tuple(dloss.shape)}, strides {dloss.stride()} do not lie "
                                 "evenly") from None
        g.dloss = dloss.data_ptr()
        dx = self._empty(x.shape, x.dtype)
        g.dx, g.ld_dx = dx.data_ptr(), d.model
        if dw is None:
            dw = self._empty(w.shape, x.dtype)
        g.grad_dtype = self._type(dw)
        g.dw, g.ld_dw = self._matrix("dw", dw, (d.vocabulary, d.model), dw.dtype)
        keep = self._workspace(d, arena_cross_entropy_backward_workspace(self.ctx, d, g))
        arena_cross_entropy_backward(self.ctx, d, g, handle)
        del keep
        return dx, dw
