"""How products are cut between their two kernels: the library's rule, compiled for the host (no GPU needed)."""

import random

import pytest

import layer_cases as cases

PAIRS = cases.HOLD[2]


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    return cases.load_cut(str(tmp_path_factory.mktemp("cut")))


@pytest.mark.parametrize("case", cases.GATED_AGAIN + cases.GATED + cases.LINEAR, ids=str)
def test_listed_cases_take_several_tiles_a_pair(cut, case):
    """What the GPU's tests of these sizes are there for: pairs of CTAs, this width, three rounds of tiles, several pieces."""
    gated, n, d_in, d_out, width = case
    pair, tokens, split, tiles, pieces = cut(n, d_in, d_out, gated)
    assert (pair, tokens, split) == (1, width, 1) and tiles > 3 * PAIRS and pieces >= 4
    assert n % width and n % 16 and d_out % 128 and -(-d_out // (128 if gated else 256)) % 12


def test_every_width_is_listed():
    """Places are three: a width counts by its turns modulo 3, of the first four warps and of the others."""
    turns = {w: ((w + 31) // 32 % 3, (w + 15) // 32 % 3) for w in range(16, 257, 16)}
    again = {w for w, (a, b) in turns.items() if 1 in (a, b)}
    assert {c[4] for c in cases.GATED_AGAIN} == again
    assert {c[4] for c in cases.GATED_AGAIN + cases.GATED} == {c[4] for c in cases.LINEAR} == set(turns)


def test_cuts_are_within_bounds(cut):
    """Any sizes, and devices that hold fewer clusters: what the kernels count on."""
    rng = random.Random(1)
    for _ in range(3000):
        n, d_in, d_out = (int(2 ** rng.uniform(0, e)) for e in (20, 16, 18))
        hold = cases.HOLD if rng.random() < 0.5 else (0, 20, 10, 6, 5, 4, 3, 2, 1)
        gated = rng.randrange(2)
        pair, tokens, split, tiles, pieces = cut(n, d_in, d_out, gated, hold)
        assert tokens % 16 == 0 and 16 <= tokens <= (256 if pair else 160)
        assert 1 <= split <= (1 if pair else min(8, pieces))
        assert pair or (tiles <= 4096 and tokens >= 2 * split)
