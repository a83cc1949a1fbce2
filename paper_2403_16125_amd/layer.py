"""Python binding of the layer operators (include/arena_layer.h): the training
step of a gated feed-forward sub-layer on the library's own kernels.

The raw functions carry the C ABI's names.  `LayerOps` wraps them for torch
tensors: it checks shapes and types, makes outputs and workspaces, and enqueues
on the current stream (or the one given).  layer_profile.py runs them together
and measures jobs for the estimator.

If the library is not built this module raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import dataclasses

from . import arena, layer_experts
from .arena import ArenaError, _check
from .layer_experts import ExpertOps, ExpertPlan

F32, BF16, F16 = 0, 1, 2
NORM_KINDS = {"rms": 0, "layer": 1}
ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}
NORM_MAX_WIDTH = 16384
# the quintic polynomial of the Muon optimiser's five steps
COEFFICIENTS = (3.4445, -4.7750, 2.0315)

EXPORTED = (
    "arena_norm_forward", "arena_norm_backward_workspace", "arena_norm_backward",
    "arena_ffn_forward_workspace", "arena_ffn_forward", "arena_ffn_backward_workspace", "arena_ffn_backward",
    "arena_orthogonal_update_workspace", "arena_orthogonal_update",
)

_i32, _i64, _f32, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class NormDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("stream_dtype", _i32), ("kind", _i32), ("width", _i32), ("tokens", _i64),
                ("gate_rows", _i64), ("eps", _f32), ("scale", _f32), ("x", _vp), ("ld_x", _i64), ("y", _vp),
                ("ld_y", _i64), ("gate", _vp), ("ld_gate", _i64), ("w_post", _vp), ("b_post", _vp), ("w_pre", _vp),
                ("b_pre", _vp), ("r", _vp), ("ld_r", _i64), ("n", _vp), ("ld_n", _i64), ("stats", _vp)]


class NormGrads(ctypes.Structure):
    _fields_ = [("dn", _vp), ("ld_dn", _i64), ("dr", _vp), ("ld_dr", _i64), ("dx", _vp), ("ld_dx", _i64),
                ("dy", _vp), ("ld_dy", _i64), ("dgate", _vp), ("dw_post", _vp), ("db_post", _vp), ("dw_pre", _vp),
                ("db_pre", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class FfnDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("activation", _i32), ("tokens", _i64), ("model", _i32), ("inner", _i32),
                ("x", _vp), ("ld_x", _i64), ("w_gate", _vp), ("ld_gate", _i64), ("w_up", _vp), ("ld_up", _i64),
                ("w_down", _vp), ("ld_down", _i64), ("g", _vp), ("u", _vp), ("h", _vp), ("ld_inner", _i64),
                ("y", _vp), ("ld_y", _i64), ("workspace", _vp), ("workspace_bytes", _i64)]


class FfnGrads(ctypes.Structure):
    _fields_ = [("grad_dtype", _i32), ("accumulate", _i32), ("dy", _vp), ("ld_dy", _i64), ("dx", _vp),
                ("ld_dx", _i64), ("dw_gate", _vp), ("ld_dw_gate", _i64), ("dw_up", _vp), ("ld_dw_up", _i64),
                ("dw_down", _vp), ("ld_dw_down", _i64)]


class UpdateDesc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("out_dtype", _i32), ("batch", _i32), ("rows", _i32), ("cols", _i32),
                ("steps", _i32), ("nesterov", _i32), ("mu", _f32), ("eps", _f32), ("scale", _f32),
                ("coefficients", _vp), ("grad", _vp), ("ld_grad", _i64), ("stride_grad", _i64), ("momentum", _vp),
                ("ld_momentum", _i64), ("stride_momentum", _i64), ("momentum_out", _vp), ("ld_momentum_out", _i64),
                ("stride_momentum_out", _i64), ("out", _vp), ("ld_out", _i64), ("stride_out", _i64),
                ("workspace", _vp), ("workspace_bytes", _i64)]


_bound = None


def load():
    """The library with the layer operators' signatures; raises if it has not been built."""
    global _bound
    lib = arena._lib
    if lib is not None and _bound is lib:
        return lib
    lib = arena.load()
    P, out = ctypes.POINTER, ctypes.POINTER(_i64)
    signatures = {
        "arena_norm_forward": [_vp, P(NormDesc), _vp],
        "arena_norm_backward_workspace": [_vp, P(NormDesc), out],
        "arena_norm_backward": [_vp, P(NormDesc), P(NormGrads), _vp],
        "arena_ffn_forward_workspace": [_vp, P(FfnDesc), out],
        "arena_ffn_forward": [_vp, P(FfnDesc), _vp],
        "arena_ffn_backward_workspace": [_vp, P(FfnDesc), P(FfnGrads), out],
        "arena_ffn_backward": [_vp, P(FfnDesc), P(FfnGrads), _vp],
        "arena_orthogonal_update_workspace": [_vp, P(UpdateDesc), out],
        "arena_orthogonal_update": [_vp, P(UpdateDesc), _vp],
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


def arena_norm_forward(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_norm_forward(ctx, _ref(desc), stream))


def arena_norm_backward_workspace(ctx, desc) -> int:
    n = _i64()
    _check(ctx, load().arena_norm_backward_workspace(ctx, _ref(desc), ctypes.byref(n)))
    return n.value


def arena_norm_backward(ctx, desc, grads, stream=0) -> None:
    _check(ctx, load().arena_norm_backward(ctx, _ref(desc), _ref(grads), stream))


def arena_ffn_forward_workspace(ctx, desc) -> int:
    n = _i64()
    _check(ctx, load().arena_ffn_forward_workspace(ctx, _ref(desc), ctypes.byref(n)))
    return n.value


def arena_ffn_forward(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_ffn_forward(ctx, _ref(desc), stream))


def arena_ffn_backward_workspace(ctx, desc, grads) -> int:
    n = _i64()
    _check(ctx, load().arena_ffn_backward_workspace(ctx, _ref(desc), _ref(grads), ctypes.byref(n)))
    return n.value


def arena_ffn_backward(ctx, desc, grads, stream=0) -> None:
    _check(ctx, load().arena_ffn_backward(ctx, _ref(desc), _ref(grads), stream))


def arena_orthogonal_update_workspace(ctx, desc) -> int:
    n = _i64()
    _check(ctx, load().arena_orthogonal_update_workspace(ctx, _ref(desc), ctypes.byref(n)))
    return n.value


def arena_orthogonal_update(ctx, desc, stream=0) -> None:
    _check(ctx, load().arena_orthogonal_update(ctx, _ref(desc), stream))


# ---------------------------------------------------------------- torch tensors

@dataclasses.dataclass
class FfnSaved:
    """What a feed-forward backward pass reads of the forward one, in one buffer:
    act(gate) * up in 16 bits, then the gate and up projections in 24, rows of
    `ld` values (a multiple of 8)."""
    buffer: object
    tokens: int
    ld: int

    def parts(self):
        """Byte offsets of h, g and u, and the buffer's size."""
        n = self.tokens * self.ld
        g = -(-2 * n // 256) * 256
        u = g + -(-3 * n // 256) * 256
        return 0, g, u, u + 3 * n


class LayerOps(ExpertOps):
    """The layer operators on one device, for torch tensors: norms around a block, the
    gated feed-forward block and the orthogonalised update here, the router, tokens to
    experts and back, the experts' blocks and the cross entropy in layer_experts.py.

    Tensors live on `device`; matrices have unit stride along their last axis
    and any row stride.  Outputs are new tensors unless given.  Work goes to the
    current stream, or to `stream`, on which the outputs and workspaces are then
    allocated."""

    _handle = None        # of the current stream, where it can be had without an object for it (1 us)

    def __init__(self, device: int = 0):
        import torch
        self.torch = torch
        self.dev = torch.device("cuda", device)
        load()
        layer_experts.load()
        self.ctx = arena.arena_create(device)
        self._alive = True
        self._index, self._new, self._current = int(device), torch.empty, torch.cuda.current_stream
        self._handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._torch_current = self._current
        self._types = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

    def close(self) -> None:
        if getattr(self, "_alive", False):
            ctx, self.ctx, self._alive = self.ctx, None, False      # later calls are refused
            arena.arena_destroy(ctx)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- checks

    def _type(self, t) -> int:
        return self._code(t.dtype)

    def _code(self, dtype) -> int:
        try:
            return self._types[dtype]
        except KeyError:
            raise ValueError(f"type {dtype} is not supported") from None

    def _matrix(self, name, t, shape, dtype):
        """Address and row stride of a 2-D tensor; a tensor of more axes is
        taken as its rows where they lie evenly."""
        if t.dtype is not dtype:
            raise ValueError(f"{name} is {t.dtype}, not {dtype}")
        if t.get_device() != self._index:
            raise ValueError(f"{name} is on {t.device}, not on {self.dev}")
        if t.dim() != 2:
            try:
                t = t.view(-1, t.shape[-1]) if t.numel() else t.reshape(-1, t.shape[-1])
            except RuntimeError:
                raise ValueError(f"{name}: the rows of shape {tuple(t.shape)}, strides {t.stride()} do not lie evenly")\
                    from None
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
        rows, cols = shape
        ld, unit = t.stride()
        if unit != 1 and cols > 1:
            raise ValueError(f"{name}: the last axis has stride {unit}, not 1")
        if ld < cols:
            if rows > 1:
                raise ValueError(f"{name}: rows overlap (stride {ld}, width {cols})")
            ld = cols
        return t.data_ptr(), ld

    def _vector(self, name, t, width, dtype):
        if t is None:
            return None
        if t.get_device() != self._index or t.dtype is not dtype or t.shape != (width,) or \
                (width > 1 and t.stride(0) != 1):
            raise ValueError(f"{name} must be a contiguous {dtype} vector of {width} on {self.dev}")
        return t.data_ptr()

    def _empty(self, shape, dtype):
        return self._new(shape, dtype=dtype, device=self.dev)

    def _workspace(self, desc, nbytes):
        """Workspace of a call: freed to the stream's pool when the caller drops it."""
        if nbytes:
            w = self._empty((nbytes,), self.torch.uint8)
            desc.workspace, desc.workspace_bytes = w.data_ptr(), nbytes
            return w
        desc.workspace, desc.workspace_bytes = None, 0
        return None

    def _run(self, stream, tensors, body, *args):
        """body(stream handle, *args), allocating on that stream.  tensors: all that
        the call is given, some of them None."""
        if self.torch.is_grad_enabled():
            for t in tensors:
                if t is not None and t.requires_grad:
                    raise ValueError(f"a tensor of shape {tuple(t.shape)} requires a gradient, which these calls do not "
                                     "record: detach it, or call under torch.no_grad()")
        # not where the host's tests, which have no GPU to ask, put a stream of their own
        if stream is None and self._handle is not None and self._current is self._torch_current:
            return body(self._handle(self._index), *args)
        current = self._current(self._index)
        if stream is None or stream == current:
            return body(current.cuda_stream, *args)
        cuda = self.torch.cuda
        outside = not cuda.is_current_stream_capturing()
        with cuda.stream(stream):
            # a stream under capture cannot wait for one outside of it
            if not (outside and cuda.is_current_stream_capturing()):
                stream.wait_stream(current)
            for t in tensors:
                if t is not None and t.is_cuda:
                    t.record_stream(stream)
            return body(stream.cuda_stream, *args)

    # -- norms around a block

    def _norm_desc(self, x_shape, dtype, stream_dtype, gate, gate_rows, scale, w_post, b_post, w_pre, b_pre, kind, eps):
        if kind not in NORM_KINDS:
            raise ValueError(f"kind must be one of {sorted(NORM_KINDS)}")
        tokens, width = x_shape
        d = NormDesc(dtype=self._code(dtype), stream_dtype=self._code(stream_dtype), kind=NORM_KINDS[kind],
                     width=width, tokens=tokens, gate_rows=int(gate_rows), eps=eps, scale=scale)
        if gate is not None:
            rows = -(-tokens // gate_rows) if gate_rows else 1
            g = gate if gate.dim() == 2 else gate.view(1, -1)
            d.gate, d.ld_gate = self._matrix("gate", g, (rows, width), dtype)
        d.w_post = self._vector("w_post", w_post, width, dtype)
        d.b_post = self._vector("b_post", b_post, width, dtype)
        d.w_pre = self._vector("w_pre", w_pre, width, dtype)
        d.b_pre = self._vector("b_pre", b_pre, width, dtype)
        return d

    @staticmethod
    def _rows(t):
        n = 1
        for v in t.shape[:-1]:
            n *= v
        return n, t.shape[-1]

    def norm_forward(self, x, y=None, *, gate=None, gate_rows=0, scale=1.0, w_post=None, b_post=None, w_pre=None,
                     b_pre=None, kind="rms", eps=1e-6, dtype=None, next_norm=True, save=False, stream=None):
        """r = x + scale * gate * norm(y; w_post, b_post) and n = norm(r; w_pre, b_pre).

        x: the residual stream [..., width], float32 or y's type; y: the
        block's output, or None (r is then x).  gate: [rows, width] or [width],
        row t // gate_rows for token t (gate_rows 0: one row).  dtype: n's type
        where y is None (x's by default).  next_norm=False leaves n out (None).
        Returns (r, n), with save=True (r, n, stats) for norm_backward."""
        return self._run(stream, (x, y, gate, w_post, b_post, w_pre, b_pre), self._norm_forward, x, y, gate, gate_rows,
                         scale, w_post, b_post, w_pre, b_pre, kind, eps, dtype, next_norm, save)

    def _norm_forward(self, handle, x, y, gate, gate_rows, scale, w_post, b_post, w_pre, b_pre, kind, eps, dtype,
                      next_norm, save):
        dtype = y.dtype if y is not None else dtype or x.dtype
        shape = self._rows(x)
        d = self._norm_desc(shape, dtype, x.dtype, gate, gate_rows, scale, w_post, b_post, w_pre, b_pre, kind, eps)
        d.x, d.ld_x = self._matrix("x", x, shape, x.dtype)
        r, n, stats = x, None, None
        if y is not None:
            d.y, d.ld_y = self._matrix("y", y, shape, dtype)
            r = self._empty(x.shape, x.dtype)
            d.r, d.ld_r = r.data_ptr(), shape[1]
        if next_norm:
            n = self._empty(x.shape, dtype)
            d.n, d.ld_n = n.data_ptr(), shape[1]
        if save:
            stats = self._empty((shape[0], 4), self.torch.float32)
            d.stats = stats.data_ptr()
        arena_norm_forward(self.ctx, d, handle)
        return (r, n, stats) if save else (r, n)

    def norm_backward(self, dn, dr, r, y, stats, *, gate=None, gate_rows=0, scale=1.0, w_post=None, b_post=None,
                      w_pre=None, b_pre=None, kind="rms", eps=1e-6, stream=None):
        """Gradients from dn and dr, those of n and r (either may be None), with
        the forward's r as it is stored (a float32 stream loses nothing there), y
        (None: no block before), stats and parameters.
        Returns a dict of dx, dy, dgate, dw_post, db_post, dw_pre and db_pre,
        None where there is no such input."""
        return self._run(stream, (dn, dr, r, y, stats, gate, w_post, b_post, w_pre, b_pre), self._norm_backward, dn, dr, r,
                         y, stats, gate, gate_rows, scale, w_post, b_post, w_pre, b_pre, kind, eps)

    def _norm_backward(self, handle, dn, dr, r, y, stats, gate, gate_rows, scale, w_post, b_post, w_pre, b_pre, kind,
                       eps):
        if dn is None and dr is None:
            raise ValueError("norm_backward needs dn or dr")
        shape = self._rows(r)
        dtype = y.dtype if y is not None else dn.dtype if dn is not None else r.dtype
        d = self._norm_desc(shape, dtype, r.dtype, gate, gate_rows, scale, w_post, b_post, w_pre, b_pre, kind, eps)
        g = NormGrads()
        p, ld = self._matrix("r", r, shape, r.dtype)
        if y is not None:
            d.y, d.ld_y = self._matrix("y", y, shape, dtype)
            d.r, d.ld_r = p, ld
        else:
            d.x, d.ld_x = p, ld
        if stats.dtype != self.torch.float32 or tuple(stats.shape) != (shape[0], 4) or not stats.is_contiguous() \
                or stats.device != self.dev:
            raise ValueError("stats is not what norm_forward saved for these tokens")
        d.stats = stats.data_ptr()
        if dn is not None:
            g.dn, g.ld_dn = self._matrix("dn", dn, shape, dtype)
        if dr is not None:
            g.dr, g.ld_dr = self._matrix("dr", dr, shape, r.dtype)
        out = dict(dx=self._empty(r.shape, r.dtype), dy=None, dgate=None, dw_post=None, db_post=None, dw_pre=None,
                   db_pre=None)
        g.dx, g.ld_dx = out["dx"].data_ptr(), shape[1]
        if y is not None:
            out["dy"] = self._empty(y.shape, dtype)
            g.dy, g.ld_dy = out["dy"].data_ptr(), shape[1]
        for name, value in (("gate", gate), ("w_post", w_post), ("b_post", b_post), ("w_pre", w_pre), ("b_pre", b_pre)):
            if value is not None:
                t = out["d" + name] = self._empty(value.shape, dtype)
                setattr(g, "d" + name, t.data_ptr())
        keep = self._workspace(g, arena_norm_backward_workspace(self.ctx, d))
        arena_norm_backward(self.ctx, d, g, handle)
        del keep
        return out

    # -- gated feed-forward block

    @staticmethod
    def _activation(name) -> int:
        if name not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
        return ACTIVATIONS[name]

    def _inner(self, tokens, inner, save):
        """A new buffer for h, with save for g and u too: FfnSaved, its address and the
        offsets of g and u."""
        saved = FfnSaved(None, tokens, -(-inner // 8) * 8)
        _, g, u, size = saved.parts()
        saved.buffer = self._empty((size if save else g,), self.torch.uint8)
        return saved, saved.buffer.data_ptr(), g, u

    def _ffn_desc(self, x, w_gate, w_up, w_down, activation):
        tokens, model = self._rows(x)
        inner = w_gate.shape[0]
        d = FfnDesc(dtype=self._type(x), activation=self._activation(activation), tokens=tokens, model=model, inner=inner)
        d.x, d.ld_x = self._matrix("x", x, (tokens, model), x.dtype)
        d.w_gate, d.ld_gate = self._matrix("w_gate", w_gate, (inner, model), x.dtype)
        d.w_up, d.ld_up = self._matrix("w_up", w_up, (inner, model), x.dtype)
        d.w_down, d.ld_down = self._matrix("w_down", w_down, (model, inner), x.dtype)
        return d

    def ffn_forward(self, x, w_gate, w_up, w_down, *, activation="silu", save=False, out=None, stream=None):
        """y = (act(x w_gate^T) * (x w_up^T)) w_down^T for x [..., model], w_gate
        and w_up [inner, model], w_down [model, inner], bfloat16 or float16.
        Returns y, with save=True (y, FfnSaved) for ffn_backward."""
        return self._run(stream, (x, w_gate, w_up, w_down, out), self._ffn_forward, x, w_gate, w_up, w_down, activation,
                         save, out)

    def _ffn_forward(self, handle, x, w_gate, w_up, w_down, activation, save, out):
        d = self._ffn_desc(x, w_gate, w_up, w_down, activation)
        y = self._empty(x.shape, x.dtype) if out is None else out
        d.y, d.ld_y = self._matrix("out", y, (d.tokens, d.model), x.dtype)
        saved, base, g, u = self._inner(d.tokens, d.inner, save)
        d.h, d.ld_inner = base, saved.ld
        if save:
            d.g, d.u = base + g, base + u
        keep = self._workspace(d, arena_ffn_forward_workspace(self.ctx, d))
        arena_ffn_forward(self.ctx, d, handle)
        del keep
        return (y, saved) if save else y

    def ffn_backward(self, dy, x, w_gate, w_up, w_down, saved, *, activation="silu", grads=None, accumulate=False,
                     stream=None):
        """(dx, dw_gate, dw_up, dw_down) from dy, with the forward's inputs and
        `saved`.  grads: three tensors for the weights' gradients, of x's type
        or float32, which accumulate=True adds to."""
        return self._run(stream, (dy, x, w_gate, w_up, w_down, saved.buffer, *(() if grads is None else grads)),
                         self._ffn_backward, dy, x, w_gate, w_up, w_down, saved, activation, grads, accumulate)

    def _ffn_backward(self, handle, dy, x, w_gate, w_up, w_down, saved, activation, grads, accumulate):
        d = self._ffn_desc(x, w_gate, w_up, w_down, activation)
        if accumulate and grads is None:
            raise ValueError("accumulate needs the gradients to add to")
        d.ld_inner = -(-d.inner // 8) * 8
        _, at_g, at_u, size = saved.parts()
        if (saved.tokens, saved.ld) != (d.tokens, d.ld_inner) or saved.buffer.numel() != size \
                or saved.buffer.device != self.dev:
            raise ValueError("saved is not what ffn_forward returned for these inputs")
        base = saved.buffer.data_ptr()
        d.h, d.g, d.u = base, base + at_g, base + at_u
        g = FfnGrads(accumulate=int(bool(accumulate)))
        g.dy, g.ld_dy = self._matrix("dy", dy, (d.tokens, d.model), x.dtype)
        dx = self._empty(x.shape, x.dtype)
        g.dx, g.ld_dx = dx.data_ptr(), d.model
        if grads is None:
            grads = tuple(self._empty(w.shape, x.dtype) for w in (w_gate, w_up, w_down))
        kind = grads[0].dtype
        g.grad_dtype = self._type(grads[0])
        g.dw_gate, g.ld_dw_gate = self._matrix("dw_gate", grads[0], (d.inner, d.model), kind)
        g.dw_up, g.ld_dw_up = self._matrix("dw_up", grads[1], (d.inner, d.model), kind)
        g.dw_down, g.ld_dw_down = self._matrix("dw_down", grads[2], (d.model, d.inner), kind)
        keep = self._workspace(d, arena_ffn_backward_workspace(self.ctx, d, g))
        arena_ffn_backward(self.ctx, d, g, handle)
        del keep
        return (dx, *grads)

    # -- orthogonalised update

    def orthogonal_update(self, grad, *, momentum=None, momentum_out=None, mu=0.95, nesterov=True,
                          coefficients=COEFFICIENTS, steps=5, eps=1e-7, scale=1.0, dtype=None, out=None, stream=None):
        """scale * (the orthogonal factor of grad, or of its momentum, by `steps`
        Newton-Schulz polynomials), for grad [rows, cols] or [batch, rows, cols].

        momentum: float32 of grad's shape, updated in place, or into
        momentum_out.  coefficients: (a, b, c) for every step, or one such triple a
        step.  dtype: of the result (bfloat16 by default, or out's)."""
        return self._run(stream, (grad, momentum, momentum_out, out), self._orthogonal_update, grad, momentum,
                         momentum_out, mu, nesterov, coefficients, steps, eps, scale, dtype, out)

    def _stack(self, name, t, shape, dtype):
        """Address, row stride and matrix stride of a tensor of two or three axes."""
        if t.device != self.dev or t.dtype != dtype or tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {self.dev}")
        rows, cols = t.shape[-2:]
        if cols > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: the last axis has stride {t.stride(-1)}, not 1")
        ld = t.stride(-2) if rows > 1 else max(cols, t.stride(-2))
        return t.data_ptr(), ld, t.stride(0) if t.dim() == 3 else 0

    def _orthogonal_update(self, handle, grad, momentum, momentum_out, mu, nesterov, coefficients, steps, eps, scale,
                           dtype, out):
        torch = self.torch
        if grad.dim() not in (2, 3):
            raise ValueError("grad must have two or three axes")
        batch = grad.shape[0] if grad.dim() == 3 else 1
        if out is None:
            out = self._empty(grad.shape, dtype or torch.bfloat16)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError(f"out is {out.dtype}, not {dtype}")
        flat = [float(v) for k in coefficients for v in (k if hasattr(k, "__len__") else (k,))]
        if len(flat) == 3 and not hasattr(coefficients[0], "__len__"):
            flat = flat * steps
        if len(flat) != 3 * steps:
            raise ValueError(f"{steps} steps need one triple of coefficients, or {steps}")
        table = (_f32 * max(1, len(flat)))(*flat)
        d = UpdateDesc(dtype=self._type(grad), out_dtype=self._type(out), batch=batch, rows=grad.shape[-2],
                       cols=grad.shape[-1], steps=steps, nesterov=int(bool(nesterov)), mu=mu, eps=eps, scale=scale)
        d.coefficients = ctypes.addressof(table)
        d.grad, d.ld_grad, d.stride_grad = self._stack("grad", grad, grad.shape, grad.dtype)
        d.out, d.ld_out, d.stride_out = self._stack("out", out, grad.shape, out.dtype)
        if momentum is not None:
            into = momentum if momentum_out is None else momentum_out
            d.momentum, d.ld_momentum, d.stride_momentum = self._stack("momentum", momentum, grad.shape, torch.float32)
            d.momentum_out, d.ld_momentum_out, d.stride_momentum_out = self._stack("momentum_out", into, grad.shape,
                                                                                   torch.float32)
        elif momentum_out is not None:
            raise ValueError("momentum_out needs momentum")
        keep = self._workspace(d, arena_orthogonal_update_workspace(self.ctx, d))
        arena_orthogonal_update(self.ctx, d, handle)
        del keep
        return out
