"""The matrices of test_muon_large_gpu.py take the ways through the products that smaller ones do not: what the
host plans for them, compiled and run here."""
import pytest

from tests.muon_plan import GRAM, NEXT, POLY, plan
from tests.test_muon_large_gpu import CALLS, PRECISE

PAIRS = 76  # that share out the units of a launch


@pytest.fixture(scope="module")
def launches():
    return [one for shapes, precise in CALLS for one in plan(shapes, PRECISE if precise else 0)]


def _matrices(launches, phase, **want):
    return [m for _, j, ms in launches if j == phase for m in ms if all(m[k] == v for k, v in want.items())]


@pytest.mark.parametrize("phase", [GRAM, POLY, NEXT])
def test_rounds(launches, phase):
    # a second unit takes the other accumulator; in B X a third the first one again, on the way there and back
    most = max(units for units, j, _ in launches if j == phase)
    assert most > (3 * PAIRS if phase == NEXT else PAIRS)


@pytest.mark.parametrize("phase", [GRAM, POLY, NEXT])
@pytest.mark.parametrize("segs", [1, 3])
def test_wide_tiles(launches, phase, segs):
    assert _matrices(launches, phase, bn=256, segs=segs, nsplit=1)


@pytest.mark.parametrize("phase,segs", [(GRAM, 1), (GRAM, 3), (POLY, 3)])
def test_wide_splits(launches, phase, segs):
    assert any(m["nsplit"] > 1 for m in _matrices(launches, phase, bn=256, segs=segs))


def test_pieces_and_mixtures(launches):
    # all of TMEM for the pieces of one unit, and half of it where a pair takes two
    assert any(m["pieces"] > 1 for u, _, ms in launches if u <= PAIRS for m in ms if m["bn"] == 256)
    assert any(m["pieces"] > 1 for u, _, ms in launches if u > PAIRS for m in ms)
    # tiles of both widths in one launch of several rounds, in both sizes of its arguments
    mixed = [len(ms) for u, _, ms in launches if u > PAIRS and {m["bn"] for m in ms} == {128, 256}]
    assert min(mixed) <= 4 < max(mixed)
    # row blocks that do not fill the last group of eight
    assert any(m["tiles_m"] > 8 and m["tiles_m"] % 8 for m in _matrices(launches, NEXT))
