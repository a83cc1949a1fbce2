"""LayerOps on a stream of the caller's choice, without a GPU: the stream waits
for the work that the inputs come from, and every tensor that the call reads or
writes there is known to the allocator as used on it."""
import contextlib
import types

import pytest

from paper_2403_16125_amd import layer


class Stream:
    def __init__(self, log, name):
        self.log, self.name, self.cuda_stream = log, name, hash(name)

    def wait_stream(self, other):
        self.log.append(f"{self.name} waits for {other.name}")

    def __eq__(self, other):
        return self.name == other.name


class Tensor:
    is_cuda, requires_grad = True, False

    def __init__(self, log, name):
        self.log, self.name = log, name

    def record_stream(self, stream):
        self.log.append(f"{self.name} used on {stream.name}")


class Rig:
    """A LayerOps whose torch only keeps a log; `capturing` names streams under capture."""

    def __init__(self):
        self.log, self.at, self.capturing = [], "main", ()
        self.ops = ops = object.__new__(layer.LayerOps)
        cuda = types.SimpleNamespace(stream=self.enter, is_current_stream_capturing=lambda: self.at in self.capturing)
        ops.torch = types.SimpleNamespace(cuda=cuda, is_grad_enabled=lambda: True)
        ops._index, ops._alive = 0, False
        ops._current = lambda device: Stream(self.log, self.at)
        for name in ("norm_forward", "norm_backward", "ffn_forward", "ffn_backward", "orthogonal_update"):
            setattr(ops, "_" + name, lambda handle, *a: self.log.append(f"launch {self.at} {handle == hash(self.at)}"))

    @contextlib.contextmanager
    def enter(self, stream):
        before, self.at = self.at, stream.name
        yield
        self.at = before

    def tensor(self, name):
        return Tensor(self.log, name)


# method, names of its tensors by position and by keyword
CALLS = {
    "norm_forward": (("x", "y"), ("gate", "w_post", "b_post", "w_pre", "b_pre")),
    "norm_backward": (("dn", "dr", "r", "y", "stats"), ("gate", "w_post", "b_post", "w_pre", "b_pre")),
    "ffn_forward": (("x", "w_gate", "w_up", "w_down"), ("out",)),
    "ffn_backward": (("dy", "x", "w_gate", "w_up", "w_down"), ()),
    "orthogonal_update": (("grad",), ("momentum", "momentum_out", "out")),
}


def call(rig, method, stream, optional=True):
    places, words = CALLS[method]
    args = [rig.tensor(n) for n in places]
    given = {n: rig.tensor(n) for n in words} if optional else {}
    names = [*places, *(words if optional else ())]
    if method == "ffn_backward":
        args.append(layer.FfnSaved(rig.tensor("saved"), 1, 8))
        names.append("saved")
        if optional:
            given["grads"] = [rig.tensor(f"grad{i}") for i in range(3)]
            names += [f"grad{i}" for i in range(3)]
    getattr(rig.ops, method)(*args, stream=stream, **given)
    return names


@pytest.mark.parametrize("method", CALLS)
@pytest.mark.parametrize("optional", [True, False])
def test_inputs_are_waited_for_and_kept(method, optional):
    rig = Rig()
    names = call(rig, method, Stream(rig.log, "side"), optional)
    at = rig.log.index("launch side True")
    assert rig.log[:at].count("side waits for main") == 1
    assert sorted(v for v in rig.log if "used on" in v) == sorted(f"{n} used on side" for n in names)


@pytest.mark.parametrize("method", CALLS)
def test_the_current_stream_needs_neither(method):
    rig = Rig()
    call(rig, method, None)
    call(rig, method, Stream(rig.log, "main"))
    assert rig.log == ["launch main True"] * 2


def test_a_captured_stream_does_not_wait_for_one_outside():
    """Such a wait would end the capture in an error; within one it forks."""
    rig = Rig()
    rig.capturing = ("side",)
    call(rig, "ffn_forward", Stream(rig.log, "side"))
    assert "side waits for main" not in rig.log and "launch side True" in rig.log
    rig.log.clear()
    rig.capturing = ("side", "main")
    call(rig, "ffn_forward", Stream(rig.log, "side"))
    assert "side waits for main" in rig.log
