"""What a decode loop over pages refuses before it begins, without a GPU."""
import types

import pytest

import seeded_inputs as si
from paper_2311_04951_amd.paged import budgeted_generate

TARGET = types.SimpleNamespace(shape=si.TINY_TARGET, max_rows=16, max_pos=64)


@pytest.mark.parametrize("changes", [dict(budget=0), dict(budget=-3), dict(keep_first=-1), dict(keep_recent=-2)])
def test_budgets_that_keep_nothing(changes):
    with pytest.raises(ValueError, match="budget"):
        budgeted_generate(TARGET, [[1, 2]], 4, 0.0, **{"budget": 8, **changes})


def test_generations_behind_the_rotary_table():
    """A prompt of n tokens and n_new of them feed n + n_new - 1 positions; the model has 64."""
    for n, n_new in ((1, 65), (60, 6), (65, 1), (66, 0), (400, 40)):
        with pytest.raises(ValueError, match="rotary"):
            budgeted_generate(TARGET, [[1, 2], [3] * n], n_new, 0.0, 8)


def test_uniforms_that_do_not_cover_the_batch():
    """The acceptance kernel reads one of every sequence a step."""
    for u in (None, [[0.5] * 4], [[0.5] * 3] * 2, [0.5] * 8):
        with pytest.raises(ValueError, match="uniforms"):
            budgeted_generate(TARGET, [[1, 2], [3]], 4, 0.8, 8, u=u)
