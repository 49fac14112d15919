"""A sequence that is released with a length past t_cap hands back the pages that a sequence can hold, and nothing of what lies behind its row in the
memory that the table is a part of."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block,t_cap", [(32, 100), (64, 256)])
def test_only_the_tables_own_entries_come_back(block, t_cap):
    from paper_2609_20888_b200 import binding as eb
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    B, most, wide = 3, -(-t_cap // block), 9
    # rows of `wide` entries, of which the table is a part that ends before the memory does
    memory = torch.full((B + 1, wide), -5, dtype=torch.int32, device="cuda")
    table = memory[:B, 2:2 + most]
    table.copy_(ints(list(range(B * most))).view(B, most))
    lens = [block * 7, 1, block * 8 + 1]
    free, n_free = ints([-1] * (4 * most)), ints([0])
    d = dict(lens=ints(lens), slots=torch.zeros(4, dtype=torch.int64, device="cuda"), pos=ints([0] * 4), start=ints([0] * (B + 1)), got=ints([0] * B),
             status=ints([0]))
    eb.eta_plan_pages(block, t_cap, ints([0, 0, 0]), d["lens"], table, free, n_free, d["slots"], d["pos"], d["start"], d["got"],
                      release=ints([1, 0, 1]), status=d["status"])
    own = list(range(most)) + list(range(2 * most, 3 * most))
    assert free.tolist() == own + [-1] * (2 * most) and n_free.tolist() == [2 * most]
    assert d["status"].tolist() == [eb.ETA_DEV_REFUSED] and d["lens"].tolist() == [0, 1, 0]
    assert d["start"].tolist() == [0, 0, 0, 0] and d["slots"].tolist() == [-1] * 4
