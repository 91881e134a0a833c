"""Decoding over pages at the ends of what it takes: budgets of a few positions, generations up to the model's last position."""
import pytest

import paper_2311_04951_amd as sv
import seeded_inputs as si
from gpu_util import weights_to_device
from paper_2311_04951_amd.paged import budgeted_generate

pytestmark = pytest.mark.gpu


def model(seed, max_pos):
    return sv.Model(si.TINY_TARGET, weights_to_device(si.decoder_weights(si.TINY_TARGET, seed)), max_rows=16, max_pos=max_pos)


@pytest.mark.parametrize("budget", [1, 2, 3, 4, 5])
def test_budgets_of_a_few_positions(budget):
    """Fewer than the first positions that are kept by default."""
    gm, stats = model(9, 256), {}
    prompts = [si.token_ids(9, f"p{i}", (n,), si.TINY_TARGET.vocab).tolist() for i, n in enumerate((40, 5))]
    got = budgeted_generate(gm, prompts, 40, 0.0, budget, page_size=16, stats=stats)
    assert stats["evictions"] >= 4 and all(len(g) == 40 for g in got)
    assert got == budgeted_generate(gm, prompts, 40, 0.0, budget, page_size=16)


def test_up_to_the_models_last_position():
    gm = model(10, 64)
    for n, n_new in ((1, 64), (60, 5), (64, 1)):
        prompt = si.token_ids(10, f"p{n}", (n,), si.TINY_TARGET.vocab).tolist()
        assert len(budgeted_generate(gm, [prompt, prompt[:1]], n_new, 0.0, 24, page_size=16)[0]) == n_new
