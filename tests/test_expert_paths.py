"""The shapes that the GPU tests check (test_gpu_expert_paths.py) take the paths that calls of
the experts' products and of the loss take: tiles, cuts and epilogues, by the library's own
choices."""
import collections
import random

import pytest

import expert_launches


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return expert_launches.build(str(tmp_path_factory.mktemp("launches")))


def paths_of(program, shapes):
    return [(at["shape"], p) for at in expert_launches.launches(program, shapes)
            for p in expert_launches.paths(at, shapes[at["shape"]])]


@pytest.fixture(scope="module")
def taken(program):
    return {p for _, p in paths_of(program, expert_launches.SHAPES)}


def test_checked_shapes_take_the_paths_of_drawn_ones(program, taken):
    rng = random.Random(2025)
    drawn = [expert_launches.draw(rng, 2e13, 1.2e9) for _ in range(8000)]
    often = collections.Counter(p for _, p in set(paths_of(program, drawn)))
    missing = sorted((n, p) for p, n in often.items() if p not in taken)
    assert not [m for m in missing if m[0] >= 4], missing
    # and all but a few of the rest
    assert len(missing) <= 0.02 * len(often), missing


@pytest.mark.parametrize("typ", [1, 2])
def test_checked_shapes_take_every_kind_of_tile(taken, typ):
    tiles = [("256", "even"), ("128", "even"), ("128", "uneven"), ("64 x 128", "even"), ("64 x 128", "uneven")]
    for kind, side in tiles:
        for call, products in (("groups", ("rows rows", "rows cols", "cols cols", "gate up", "gate up back")),
                               ("loss", ("logits", "logits back", "rows cols"))):
            for product in products:
                assert any(p[:5] == (call, product, typ, kind, side) for p in taken), (call, product, kind, side)
                if product.startswith("gate up"):
                    for act in range(3):
                        assert any(p[:5] == (call, product, typ, kind, side) and p[6:] == ("activation", act)
                                   for p in taken), (product, kind, side, act)
        for product in ("rows rows", "rows cols"):
            assert ("groups", product, typ, kind, side, "whole") in taken
    for kind in ("128", "64 x 128"):
        for side in ("even", "uneven"):
            for product in ("rows rows", "rows cols", "gate up back"):
                assert ("groups", product, typ, kind, side, "split") in taken, (product, kind, side)
    assert any(p[2:4] == (typ, "streamed") for p in taken)
    for product in ("rows rows", "rows cols"):
        parts = {p[3:5] for p in taken if p[:3] == ("groups", product, typ) and p[-1] == "last round in parts"}
        assert ("128", "even") in parts and ("128", "uneven") in parts, (product, parts)
