"""LayerOps does not record gradients: inputs that ask for one are refused, not
answered with tensors that silently lack it.  Needs no GPU: the check comes first."""
import types

import pytest
import torch

from paper_2403_16125_amd import layer


@pytest.fixture(scope="module")
def ops():
    o = layer.LayerOps()
    o._current = lambda device: types.SimpleNamespace(cuda_stream=0)
    for name in ("norm_forward", "norm_backward", "ffn_forward", "ffn_backward", "orthogonal_update"):
        setattr(o, "_" + name, lambda handle, *a: "ran")
    yield o
    o.close()


def leaf(grad):
    return torch.zeros(4, 4, requires_grad=grad)


CALLS = [("norm_forward", ("x", "y"), ("gate", "w_post", "b_post", "w_pre", "b_pre")),
         ("norm_backward", ("dn", "dr", "r", "y", "stats"), ("gate", "w_post", "b_post", "w_pre", "b_pre")),
         ("ffn_forward", ("x", "w_gate", "w_up", "w_down"), ("out",)),
         ("ffn_backward", ("dy", "x", "w_gate", "w_up", "w_down", "saved"), ("grads",)),
         ("orthogonal_update", ("grad",), ("momentum", "momentum_out", "out"))]


def run(ops, method, places, words, which, requires=True):
    def make(name):
        if name == "saved":
            return layer.FfnSaved(torch.zeros(8), 1, 8)
        if name == "grads":
            return [leaf(False), leaf(requires and which == name), leaf(False)]
        return leaf(requires and which == name)
    return getattr(ops, method)(*(make(n) for n in places), **{n: make(n) for n in words})


@pytest.mark.parametrize("method,places,words,which",
                         [(m, p, w, n) for m, p, w in CALLS for n in p + w if n != "saved"])
def test_inputs_that_require_a_gradient_are_refused(ops, method, places, words, which):
    with pytest.raises(ValueError, match="requires a gradient"):
        run(ops, method, places, words, which)
    assert run(ops, method, places, words, which, requires=False) == "ran"
    with torch.no_grad():
        assert run(ops, method, places, words, which) == "ran"
    with torch.inference_mode():
        assert run(ops, method, places, words, which) == "ran"
