"""Items, and halves of items, that see nothing, among others that do, on the same CTA: what the two threads of a row tell each other belongs to one item."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_prefill import DENSE, CANARY, call, check, ints, make, workspace
from test_gpu_prefill_past_length import many_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("paged", [False, True])
def test_sequences_that_see_nothing_between_others(gated, paged):
    """Enough of them that every CTA has several items; halves without tiles where fewer rows than a half see something."""
    rows, lens = [70, 90, 33, 64, 128] * 40, [70, 5, 0, 20, 200] * 40
    s = many_rows(rows, lens, 2, 4, 64, 32, paged, seed=41)
    params, const = (eb.DecodeParams(), torch.full((8,), 0.2, device="cuda")) if gated else (DENSE, None)
    out = check(s, params, const=const, status=eb.ETA_DEV_EMPTY_ROW)
    for _ in range(10):
        assert torch.equal(call(s, params, const=const)[0], out)


def test_shares_that_hold_the_last_tile_of_a_half_only():
    """Split items whose last part has a tile that only the second half sees: 64 tokens an item, the second 32 of which begin a tile."""
    new, before = [64] * 24, [8160 + 128 * k for k in range(24)]          # the last 32 tokens stand in a tile of their own
    s = make(new, before, 1, 4, 128, 64, True, seed=42)
    out = check(s, DENSE)
    desc = eb.paged_cache_desc(s["K"], s["V"], s["B"], s["Hq"], t_cap=s["NB"] * s["b"])
    pages, ws, starts, lens = eb.page_table(s["table"], s["K"].shape[0]), workspace(desc), ints(s["starts"]), ints(s["lens"])
    outs = [torch.full_like(out, CANARY) for _ in range(30)]
    for o in outs:
        eb.eta_prefill(desc, DENSE, s["q"], s["K"], s["V"], starts, lens, o, ws, pages=pages)
    assert all(torch.equal(o, out) for o in outs)
