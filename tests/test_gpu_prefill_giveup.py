"""Bounded waits of prompt attention that run out, on purpose, without faulting or hanging anything.

A build of the same sources (-DETA_TEST_SKIP_WEIGHTS_ARRIVE -DETA_TEST_SKIP_LAST_COMMIT -DETA_WAIT_LIMIT=65536) in which a softmax warp of the first CTA's second half never says that
its weights are there, with waits of 2^16 polls (a few milliseconds: far longer than a copy or a product takes).  The warp that issues the products
gives up, and everyone who waits for it; halves of the CTA may be at different items then, one of them at an item that both would work on.  And
in the second CTA the last product of an item for one half is never announced: the copies and the products are all done by the time that the softmax warps
give up.
Checked: the call returns and reports ETA_DEV_TIMEOUT, rows of other CTAs are as ever, and an ordinary call on the same buffers right afterwards is correct."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_prefill import CANARY, DENSE, call, make, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def variant():
    from paper_2609_20888_b200 import build as ebuild
    ebuild.build()
    eb.load()
    return eb.load(ebuild.build_giveup_variant())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("new,before,whole", [([300], [0], False), ([1] * 3, [3000] * 3, False), ([40, 1] * 150, [200, 300] * 150, True),
                                              ([64, 1, 1], [2000, 3000, 3000], False)])
def test_weights_that_never_come_end_in_a_timeout(variant, monkeypatch, new, before, whole, gated):
    s = make(new, before, 1, 4, 64, 64, False, seed=51)
    params, const = (eb.DecodeParams(), torch.full((4,), 0.2, device="cuda")) if gated else (DENSE, None)
    want, status = call(s, params, const=const)
    assert status == 0
    ws = workspace(eb.cache_desc(s["K"], s["V"], s["Hq"], s["b"]))
    out = torch.full_like(want, CANARY)
    with monkeypatch.context() as m:
        m.setattr(eb, "_lib", variant)
        _, status = call(s, params, const=const, out=out, ws=ws)
    torch.cuda.synchronize()
    assert status == eb.ETA_DEV_TIMEOUT, "the wait did not run out, or did not report it"
    if whole:
        # items go to the CTAs in rounds, back and forth: of 300 the first CTA has the first and one more; most are others'
        same = torch.tensor([torch.equal(out[a:b], want[a:b]) for a, b in zip(s["starts"], s["starts"][1:])])
        assert (~same).sum() <= 3
    again, status = call(s, params, const=const, out=out, ws=ws)
    assert status == 0 and torch.equal(again, want)


@pytest.mark.parametrize("gated", [False, True])
def test_a_last_product_that_never_comes_is_reported(variant, monkeypatch, gated):
    """A hundred single tokens of a tile each, an item a CTA."""
    s = make([1] * 100, [i for i in range(20, 120)], 1, 4, 64, 64, False, seed=52)
    params, const = (eb.DecodeParams(), torch.full((4,), 0.2, device="cuda")) if gated else (DENSE, None)
    want, status = call(s, params, const=const)
    assert status == 0
    out, ws = torch.full_like(want, CANARY), workspace(eb.cache_desc(s["K"], s["V"], s["Hq"], s["b"]))
    with monkeypatch.context() as m:
        m.setattr(eb, "_lib", variant)
        _, status = call(s, params, const=const, out=out, ws=ws)
    assert status == eb.ETA_DEV_TIMEOUT
    assert torch.equal(out[:1], want[:1]) and torch.all(out[1] == CANARY) and torch.equal(out[2:], want[2:])
    again, status = call(s, params, const=const, out=out, ws=ws)
    assert status == 0 and torch.equal(again, want)
