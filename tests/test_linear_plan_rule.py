"""Which tile bpe_linear takes, restated (linear_plan.py) and compared with what the library asks for as workspace; and that the
sizes which the GPU tests run reach every tile, whole and in parts.  No GPU is needed."""
import math
import random

import linear_cases
import linear_plan
import pytest


@pytest.fixture(scope="module", autouse=True)
def _read_once():
    rows, read = linear_plan.tiles(), linear_plan.tiles
    linear_plan.tiles = lambda: rows
    yield
    linear_plan.tiles = read


def test_the_restated_rule_asks_for_the_same_workspace():
    import paper_2603_02597_amd as B
    rng = random.Random(1)

    def size(low, high):
        return int(math.exp(rng.uniform(math.log(low), math.log(high))))

    split = 0
    for _ in range(5000):
        m, n, k = size(1, 9000), size(1, 130000), size(1, 9000)
        want = linear_plan.workspace_bytes(m, n, k)
        assert B.bpe_linear_workspace_bytes(m, n, k) == want, (m, n, k)
        split += want > 0
    assert 500 < split < 4500


def test_the_cases_reach_what_they_say():
    for tile, parts, m, n, k in linear_cases.CASES:
        for aligned in (True, False):
            got, splits = linear_plan.plan(m, n, k, aligned)
            assert (got, splits > 1) == (tile, parts), (m, n, k)


def test_the_cases_reach_every_tile():
    assert len(linear_plan.tiles()) == 6
    assert {(tile, parts) for tile, parts, *_ in linear_cases.CASES} == {(t, parts) for t in range(6) for parts in (False, True)}
