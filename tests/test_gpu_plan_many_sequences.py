"""Steps of so many sequences without new tokens that the rows of a CTA lie between more row starts than it keeps in shared memory."""
import pytest
import torch

from tests.test_gpu_plan_pages import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows_behind", [0, 1, 2000])
@pytest.mark.parametrize("batch", [3001, 9000])
def test_prompts_far_apart_among_idle_sequences(batch, rows_behind):
    g = torch.Generator().manual_seed(batch)
    new = [0] * batch
    for i in torch.randperm(batch, generator=g)[:12].tolist():
        new[i] = int(torch.randint(200, 700, (1,), generator=g))
    new[0], new[batch - 1] = 5, 3                              # (the idle ones lie between rows of one CTA too)
    lens = torch.randint(0, 100, (batch,), generator=g).tolist()
    check(32, 1024, new, lens, 32, 4 * batch, max(4097, sum(new)) + rows_behind, seed=batch, in_place=True)


def test_all_idle_and_one_prompt_at_the_end():
    lens, new = [40] * 5000, [0] * 4999 + [5000]
    check(64, 6400, new, lens, 100, 6000, 5000)
    check(64, 6400, [-1] * 5000, lens, 100, 6000, 5000)
