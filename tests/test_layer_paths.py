"""The shapes that the GPU tests check take the paths that calls take: tiles, cuts
and epilogues, by the library's own choices."""
import collections
import random

import pytest

import layer_launches


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return layer_launches.build(str(tmp_path_factory.mktemp("launches")))


def paths_of(program, shapes):
    return [(launch["shape"], p) for launch in layer_launches.launches(program, shapes) for p in layer_launches.paths(launch)]


def test_checked_shapes_take_the_paths_of_drawn_ones(program):
    rng = random.Random(2024)
    drawn = [layer_launches.draw(rng, 7e12) for _ in range(5000)]
    taken = {p for _, p in paths_of(program, layer_launches.SHAPES)}
    often = collections.Counter(p for _, p in set(paths_of(program, drawn)))
    missing = sorted((n, p) for p, n in often.items() if p not in taken)
    assert not [m for m in missing if m[0] >= 4], missing
    # and all but a few of the rest
    assert len(missing) <= 0.05 * len(often), missing


def test_checked_shapes_take_every_kind_of_tile(program):
    """Each product's tiles, whole rounds before smaller ones, and mirrored tiles of each kind."""
    taken = {p for _, p in paths_of(program, layer_launches.SHAPES)}
    for product in ("rows rows", "rows cols", "cols cols", "gate up", "gate up back"):
        for typ in (1, 2):
            for tile in ("256", "128", "128 deep", "64"):
                assert any(p[:2] == (product, typ) and tile in p[2:3] for p in taken), (product, typ, tile)
    for product in ("rows rows rest", "rows cols rest"):
        for tile in ("256", "128", "128 deep", "64"):
            assert any(p[:3] == (product, 2, tile) for p in taken), (product, tile)
    for tile in ("256", "128", "128 deep", "64"):
        assert any(p[2] == tile and "mirrored" in p and "split" not in p for p in taken), tile
    assert any("after whole rounds" in p and "smaller tiles" in p and "split" in p and "mirrored" in p for p in taken)
    assert any("after whole rounds" in p and "unsplit" in p and "mirrored" in p for p in taken)
