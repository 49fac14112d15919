"""Negative counts of holders count as 0: what forks, releases and compaction make of them is what they make of zeros."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_page_sharing import SIZES, Pool, ints, workspace

pytestmark = pytest.mark.gpu


def program(size, in_place, negative):
    """Fork, release of parents, compaction, a plan for the next tokens -> everything that the calls left behind."""
    block, stride, lens, n_pages = SIZES[size]
    p = Pool(block, stride, lens, n_pages, seed=71)
    t = p.tensors()
    if negative:
        gen = torch.Generator().manual_seed(72)
        t["shared"] = torch.where(t["shared"] == 0, -torch.randint(1, 5, (n_pages,), generator=gen, dtype=torch.int32).cuda(), t["shared"])
        if negative > 1:
            t["shared"][::3] = -2 ** 31
    B, cap = len(lens), block * stride
    whole = [i for i, n in enumerate(lens) if n > 0]
    parent = ints([whole[(3 * i) % len(whole)] if n == 0 else -1 for i, n in enumerate(lens)])
    src, dst, granted, status, kept = ints([0] * B), ints([0] * B), ints([0] * B), ints([0]), []

    def out(name):
        if in_place:
            return None
        return torch.full_like(t[name], 77)

    def take(**new):
        for k, v in new.items():
            if v is not None:
                t[k] = v
        kept.extend((t["shared"].clamp(min=0), t["lens"].clone(), t["table"].clone(), t["n_free"].clone(), t["free"].clone()))

    o = {k: out(k) for k in ("lens", "shared", "n_free")}
    eb.eta_fork_pages(block, cap, parent, t["lens"], t["table"], t["shared"], t["free"], t["n_free"], src, dst, granted, seq_lens_out=o["lens"],
                      shared_out=o["shared"], n_free_out=o["n_free"], status=status)
    take(**o)
    kept.extend((src, dst, granted))
    o, ws = {k: out(k) for k in ("lens", "shared", "n_free")}, workspace(n_pages)
    eb.eta_free_pages(block, cap, ints([int(n > 0) for n in lens]), t["lens"], t["table"], t["shared"], t["free"], t["n_free"], ws, seq_lens_out=o["lens"],
                      shared_out=o["shared"], n_free_out=o["n_free"], status=status)
    take(**o)
    # no page of a child is on the stack
    stack = set(t["free"][:int(t["n_free"])].tolist())
    for i, n in enumerate(t["lens"].tolist()):
        assert not stack & set(t["table"][i, :-(-n // block)].tolist())
    if negative:
        t["shared"] = torch.where(t["shared"] == 0, -1, t["shared"])
    moves = [ints([5] * n_pages), ints([5] * n_pages), ints([0])]
    o = {k: out(k) for k in ("table", "shared", "n_free")}
    free_out = t["free"].clone()
    eb.eta_compact_pages(block, cap, t["lens"], t["table"], t["shared"], t["free"], t["n_free"], *moves, ws, block_table_out=o["table"],
                         shared_out=o["shared"], free_pages_out=None if in_place else free_out, n_free_out=o["n_free"], status=status)
    if not in_place:
        assert (o["shared"] >= 0).all()
        # (entries of a table's row behind its sequence are copied, too)
        t["free"] = free_out
    take(**o)
    kept.extend(moves)
    room = ints([min(1, cap - n) if n else 0 for n in t["lens"].tolist()])
    slots, start = torch.zeros(B, dtype=torch.int64, device="cuda"), ints([0] * (B + 1))
    eb.eta_plan_pages(block, cap, room, t["lens"], t["table"], t["free"], t["n_free"], slots, ints([0] * B), start, granted, status=status)
    kept.extend((slots, t["table"], granted))
    return [x.tolist() for x in kept], int(status)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("negative", [1, 2])
@pytest.mark.parametrize("size", list(SIZES))
def test_negative_counts_are_zeros(size, in_place, negative):
    assert program(size, in_place, negative) == program(size, in_place, 0)
