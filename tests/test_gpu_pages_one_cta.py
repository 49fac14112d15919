"""The calls on pages of large pools by one CTA, as on a GPU that holds no cluster of eight: a build of the library that takes that way whatever the size gives
what the product library gives."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_page_sharing import SIZES, Pool, run_compact, run_fork, run_release

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("size", ["large", "wide"])
def test_large_pools(monkeypatch, size, in_place):
    from paper_2609_20888_b200 import build as ebuild
    ebuild.build()
    eb.load()
    monkeypatch.setattr(eb, "_lib", eb.load(ebuild.build_general_variant()))
    block, stride, lens, n_pages = SIZES[size]
    p = Pool(block, stride, lens, n_pages, seed=101)
    whole = [i for i, n in enumerate(lens) if n > 0]
    run_fork(p, [whole[(3 * i) % len(whole)] if n == 0 else -1 for i, n in enumerate(lens)], None, in_place)
    run_release(p, [int(i % 3 == 0) for i in range(len(lens))], in_place)
    run_compact(p, in_place)
    run_release(p, [1] * len(lens), in_place)
    assert p.n_free == n_pages and not any(p.shared)
    torch.cuda.synchronize()
