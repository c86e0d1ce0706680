"""The sizes by which the linear layer's products are tested choose every tile, whole and divided, even and with ends."""
import shutil

import pytest

from layer_plans import FORWARD, INPUT, WEIGHT, Plans
from layer_sizes import SIZES, cases

CALLS = {FORWARD: [(256, 256), (128, 128), (256, 32)], INPUT: [(256, 256), (256, 128), (128, 128), (256, 32)], WEIGHT: [(256, 256), (128, 128)]}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    return Plans(str(tmp_path_factory.mktemp("plans")))


def test_every_tile_and_type_is_listed(plans):
    want = {(c, tile, t) for c, tiles in CALLS.items() for tile in tiles for t in ((None,) if c == FORWARD else ("bf16", "f16", "f32"))}
    assert set(SIZES) == want and all(len(v) == 4 for v in SIZES.values())
    # no tile but these is chosen: over the sizes' range, a grid of them
    found = {c: set() for c in CALLS}
    for c in CALLS:
        for t in ("bf16", "f16", "f32"):
            for rows in (1, 17, 40, 130, 700, 2049, 9000):
                for n_in in (1, 100, 900, 5000, 16384):
                    for n_out in (1, 100, 900, 5000, 16384):
                        p = plans.divide(c, t, rows, n_in, n_out)
                        found[c].add((p["ti"], p["to"]))
    assert found == {c: set(tiles) for c, tiles in CALLS.items()}


@pytest.mark.parametrize("call", list(CALLS))
def test_sizes_choose_what_they_stand_for(plans, call):
    by_piece, later_planes, turns = set(), set(), set()
    for tile, t, divided, ragged, (rows, n_in, n_out) in cases(call):
        p = plans.divide(call, t or "bf16", rows, n_in, n_out)
        assert (p["ti"], p["to"]) == tile and (p["pieces"] > 1) == divided, (call, tile, t, divided, ragged, p)
        inner, outer = {FORWARD: (n_out, rows), INPUT: (n_in, rows), WEIGHT: (n_in, n_out)}[call]
        assert bool(inner % tile[0]) == bool(outer % tile[1]) == ragged
        last = p["steps"] - p["per"] * (p["pieces"] - 1)
        assert min(p["per"], last) >= 9
        by_piece.add((divided, p["by_piece"]))
        plane = p["steps"] // p["planes"]
        for s0 in range(0, p["steps"], p["per"]):
            if s0 // plane:
                later_planes.add((t, s0 // plane))          # pieces that start in it
            if s0 // plane != (min(s0 + p["per"], p["steps"]) - 1) // plane:
                turns.add(t)                                # pieces that go on from one plane into the next
    assert by_piece >= {(1, 0), (1, 1)}                     # divided sums by dies and spread over them
    if call != FORWARD:
        assert later_planes == {("f16", 1), ("f32", 1), ("f32", 2)} and turns == {"f16", "f32"}
