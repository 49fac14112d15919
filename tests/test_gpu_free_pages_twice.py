"""Releases of pages that nobody holds: they are on the stack already and do not go there again."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_page_sharing import Pool, ints, workspace

pytestmark = pytest.mark.gpu

SIZES = {"one CTA": (64, 6, [200, 384, 64, 0, 130], 30), "a cluster": (64, 150, [9000, 0, 4096, 9600, 63] * 8, 4001)}


def release(p, t, which, in_place, ws):
    o = {k: None if in_place else torch.full_like(t[k], 77) for k in ("lens", "shared", "n_free")}
    status = ints([0])
    eb.eta_free_pages(p.block, p.stride * p.block, ints(which), t["lens"], t["table"], t["shared"], t["free"], t["n_free"], ws, seq_lens_out=o["lens"],
                      shared_out=o["shared"], n_free_out=o["n_free"], status=status)
    t.update({k: v for k, v in o.items() if v is not None})
    return int(status)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("size", list(SIZES))
def test_a_second_release(size, in_place):
    block, stride, lens, n_pages = SIZES[size]
    p = Pool(block, stride, lens, n_pages, seed=91)
    t, ws = p.tensors(), workspace(n_pages)
    gone = [int(i % 2 == 0) for i in range(len(lens))]
    assert release(p, t, gone, in_place, ws) == 0
    once = {k: v.clone() for k, v in t.items()}
    # the same sequences again, their lengths as before: all of their pages are free
    t["lens"] = ints(lens)
    assert release(p, t, gone, in_place, ws) == eb.ETA_DEV_REFUSED
    assert all(torch.equal(t[k], once[k]) for k in t)
    # beside the others: only the pages that they hold come back
    t["lens"] = ints(lens)
    assert release(p, t, [1] * len(lens), in_place, ws) == eb.ETA_DEV_REFUSED
    assert int(t["n_free"]) == n_pages and sorted(t["free"].tolist()) == list(range(n_pages)) and not t["shared"].any()


@pytest.mark.parametrize("size", list(SIZES))
def test_a_stack_of_numbers_that_are_no_pages(size):
    """They are left where they are; what else the workspace holds of them does not matter."""
    block, stride, lens, n_pages = SIZES[size]
    p = Pool(block, stride, lens, n_pages, seed=92)
    p.free[:3] = [-1, n_pages, 2 ** 31 - 1]
    t = p.tensors()
    held = sorted(p.table[0][:-(-lens[0] // block)])
    assert release(p, t, [1] + [0] * (len(lens) - 1), True, workspace(n_pages)) == 0
    assert t["free"].tolist() == p.free[:p.n_free] + held + p.free[p.n_free + len(held):] and int(t["n_free"]) == p.n_free + len(held)


def test_whatever_the_workspace_holds():
    """A workspace full of numbers below the stack's height: a page counts as free only where the stack says so."""
    p = Pool(64, 6, [200, 384, 64, 0, 130], 30, seed=93)
    for fill in (0, 1, 5):
        t, ws = p.tensors(), workspace(30)
        ws.view(torch.int32).fill_(fill)
        assert release(p, t, [1, 1, 1, 1, 1], True, ws) == 0
        assert int(t["n_free"]) == 30 and sorted(t["free"].tolist()) == list(range(30))
