"""Forks where a table or the stack holds numbers that are no pages: a child whose copy cannot be made is turned away, not served without its last tokens."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_page_sharing import Pool, ints

pytestmark = pytest.mark.gpu

SIZES = {"one CTA": (64, 6, 40), "a cluster": (64, 6, 5000)}


def fork(p, parent):
    t = p.tensors()
    B = len(parent)
    src, dst, granted, status = ints([55] * B), ints([55] * B), ints([55] * B), ints([0])
    eb.eta_fork_pages(p.block, p.stride * p.block, ints(parent), t["lens"], t["table"], t["shared"], t["free"], t["n_free"], src, dst, granted,
                      status=status)
    return t, src.tolist(), dst.tolist(), granted.tolist(), int(status)


@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("bad", [-1, -2 ** 31, "n_pages", 1 << 30, 2 ** 31 - 1])
def test_a_parents_last_page(size, bad):
    block, stride, n_pages = SIZES[size]
    p = Pool(block, stride, [200, 0, 0, 130, 0, 0], n_pages, seed=81)
    whole, top = list(p.table[3][:2]), p.free[:p.n_free]
    p.table[0][3] = n_pages if bad == "n_pages" else bad
    last = p.table[3][2]
    t, src, dst, granted, status = fork(p, [-1, 0, 3, -1, 0, 3])
    assert status == eb.ETA_DEV_REFUSED and granted == [0, 0, 130, 0, 0, 130]
    assert t["lens"].tolist() == [200, 0, 130, 130, 0, 130]
    # the children that are turned away take no page off the stack
    assert src == [-1, -1, last, -1, -1, last] and dst == [-1, -1, top[-1], -1, -1, top[-2]] and int(t["n_free"]) == p.n_free - 2
    want = [list(r) for r in p.table]
    want[2][:3], want[5][:3] = whole + [top[-1]], whole + [top[-2]]
    assert t["table"].tolist() == want
    assert [t["shared"][x].item() for x in whole] == [2, 2] and int(t["shared"].sum()) == 4


@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("bad", [-9, "n_pages", 1 << 30])
def test_a_number_on_the_stack(size, bad):
    block, stride, n_pages = SIZES[size]
    p = Pool(block, stride, [130, 0, 0, 128, 0, 0], n_pages, seed=82)
    p.free[p.n_free - 2] = n_pages if bad == "n_pages" else bad
    top, last = p.free[:p.n_free], p.table[0][2]
    t, src, dst, granted, status = fork(p, [-1, 0, 0, -1, 3, 0])
    # the second child that wants a page would get it; the number is off the stack then, too
    assert status == eb.ETA_DEV_REFUSED and granted == [0, 130, 0, 0, 128, 130]
    assert src == [-1, last, -1, -1, -1, last] and dst == [-1, top[-1], -1, -1, -1, top[-3]] and int(t["n_free"]) == p.n_free - 3
    assert t["lens"].tolist() == [130, 130, 0, 128, 128, 130] and t["table"][2].tolist() == p.table[2]
    assert [t["shared"][x].item() for x in p.table[0][:2]] == [2, 2] and [t["shared"][x].item() for x in p.table[3][:2]] == [1, 1]


@pytest.mark.parametrize("size", list(SIZES))
def test_a_full_page_is_handed_on_and_said(size):
    block, stride, n_pages = SIZES[size]
    p = Pool(block, stride, [256, 0, 0], n_pages, seed=83)
    p.table[0][1] = n_pages + 7
    t, src, dst, granted, status = fork(p, [-1, 0, 0])
    assert status == eb.ETA_DEV_REFUSED and granted == [0, 256, 256]
    assert t["table"][1].tolist()[:4] == p.table[0][:4] == t["table"][2].tolist()[:4]
    assert int(t["shared"].sum()) == 6 and (t["shared"][[p.table[0][k] for k in (0, 2, 3)]] == 2).all()
