"""The tables of tests/wgrad_tile_cases.py take the side and the shares that they are there for: where a changed estimate moves
one, it has to be replaced by one that does, or a kernel is left without a test."""
import pytest

from tests.grad_plan_program import WEIGHT_GRAD, program, schedule
from tests.wgrad_tile_cases import CASES


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    return program(tmp_path_factory.mktemp("plan"), WEIGHT_GRAD)


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_side_and_shares(run, name, accumulate):
    dtype, side, whole, split, layers = CASES[name]
    p = schedule(run, [(t, o, i, o + gap, n + 1) for n, (t, o, i, gap) in enumerate(layers)], int(dtype == "bf16"), accumulate)
    assert (p.tile, p.whole > 0, p.tiles > p.whole) == (side, whole, split)
    assert not split or p.split > 1


def test_every_way_is_reached():
    for dtype in ("bf16", "f32"):
        for side, whole, split in ((256, True, False), (256, False, True), (256, True, True), (128, True, True)):
            assert any(c[:4] == (dtype, side, whole, split) for c in CASES.values())
    assert any(len(c[4]) > 1 for c in CASES.values())
