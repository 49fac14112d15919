"""Forks, release, compaction and copies of pages refuse on the host what they cannot do: no device is touched."""
import ctypes

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild

ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)


@pytest.fixture(scope="module")
def lib():
    ebuild.build()
    return eb.load()


ORDERS = {
    "eta_fork_pages": "batch block_size t_cap parent take seq_lens seq_lens_out table stride shared shared_out free n_free n_free_out n_pages "
                      "copy_src copy_dst granted status stream",
    "eta_free_pages": "batch block_size t_cap release seq_lens seq_lens_out table stride shared shared_out free n_free n_free_out n_pages status "
                      "ws ws_bytes stream",
    "eta_compact_pages": "batch block_size t_cap seq_lens table table_out stride shared shared_out free free_out n_free n_free_out n_pages move_src "
                         "move_dst n_moves status ws ws_bytes stream",
}


def _call(lib, name, **kw):
    args = dict.fromkeys(ORDERS[name].split(), ONE)
    args.update(batch=2, block_size=64, t_cap=4096, stride=64, n_pages=128, status=None, stream=None, take=None, ws_bytes=1 << 30)
    args.update(kw)
    return getattr(lib, name)(*(args[k] for k in ORDERS[name].split()))


@pytest.mark.parametrize("name", list(ORDERS))
@pytest.mark.parametrize("kw,code", [(dict(batch=0), -1), (dict(block_size=48), -2), (dict(t_cap=0), -1), (dict(stride=63), -1), (dict(n_pages=0), -1),
                                     (dict(n_pages=(1 << 30) + 1), -2), (dict(batch=(1 << 30) + 1), -2)])
def test_sizes(lib, name, kw, code):
    assert _call(lib, name, **kw) == code


@pytest.mark.parametrize("name,missing", [(name, k) for name in ORDERS for k in ORDERS[name].split()
                                          if k not in "batch block_size t_cap stride n_pages status stream take ws ws_bytes".split()])
def test_missing_arrays(lib, name, missing):
    assert _call(lib, name, **{missing: None}) == -1


@pytest.mark.parametrize("name", ["eta_free_pages", "eta_compact_pages"])
@pytest.mark.parametrize("kw", [dict(ws=None), dict(ws=ODD), dict(ws_bytes=100)])
def test_workspace(lib, name, kw):
    assert _call(lib, name, **kw) == -3


def test_a_fork_takes_1024_sequences(lib):
    assert _call(lib, "eta_fork_pages", batch=1025) == -2


def test_workspace_bytes(lib):
    n = eb.eta_pages_workspace_bytes(1000)
    assert n % 256 == 0 and n >= 4000
    assert eb.eta_pages_workspace_bytes(1 << 20) > 4 << 20
    size = ctypes.c_size_t(0)
    assert lib.eta_pages_workspace_bytes(0, ctypes.byref(size)) == -1 and lib.eta_pages_workspace_bytes(5, None) == -1


def _pool(**kw):
    return eb.PagePool(**{**dict(base=256, page_stride=4096, piece_stride=0, piece_bytes=4096, n_pieces=1), **kw})


@pytest.mark.parametrize("pool,code", [(_pool(base=None), -1), (_pool(base=264), -2), (_pool(n_pieces=0), -1), (_pool(piece_bytes=0), -1),
                                       (_pool(page_stride=0), -1), (_pool(page_stride=4104), -2), (_pool(piece_bytes=40), -2),
                                       (_pool(n_pieces=2, piece_stride=8), -2), (_pool(n_pieces=2, piece_stride=16), -1),
                                       (_pool(piece_bytes=1 << 50), -2)])
def test_pools(lib, pool, code):
    assert lib.eta_copy_pages(ctypes.byref(pool), 1, 10, ONE, ONE, 5, None, None, None) == code


def test_copy_arguments(lib):
    p = _pool()
    assert lib.eta_copy_pages(None, 1, 10, ONE, ONE, 5, None, None, None) == -1
    assert lib.eta_copy_pages(ctypes.byref(p), 0, 10, ONE, ONE, 5, None, None, None) == -1
    assert lib.eta_copy_pages(ctypes.byref(p), 1, 0, ONE, ONE, 5, None, None, None) == -1
    assert lib.eta_copy_pages(ctypes.byref(p), 1, 10, None, ONE, 5, None, None, None) == -1
    assert lib.eta_copy_pages(ctypes.byref(p), 1, 10, ONE, ONE, -1, None, None, None) == -1
    assert lib.eta_copy_pages((eb.PagePool * 65)(*[p] * 65), 65, 10, ONE, ONE, 5, None, None, None) == -2
    assert lib.eta_copy_pages(ctypes.byref(p), 1, 10, None, None, 0, None, None, None) == 0


@pytest.mark.parametrize("kw,code", [(dict(desc=None), -1), (dict(parent=None), -1), (dict(granted=None), -1), (dict(musig=None), -1),
                                     (dict(mnorm=None), -1), (dict(musig=ODD), -2), (dict(flags=1), -1)])
def test_fork_summaries(lib, kw, code):
    d = eb.CacheDesc(2, 8, 2, 128, 64, 4096, 64, 0, 0, 0, 0, 0, 0)
    a = {**dict(desc=ctypes.byref(d), parent=ONE, granted=ONE, musig=ONE, mnorm=ONE, flags=0), **kw}
    assert lib.eta_fork_summaries(a["desc"], a["parent"], a["granted"], a["musig"], a["mnorm"], a["flags"], None, None) == code


def test_cpu_tensors_are_refused():
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(eb.EtaError):
        eb.eta_copy_pages([torch.zeros(4, 64)], t, t)
    with pytest.raises(eb.EtaError):
        eb.eta_copy_pages([], t, t)
    with pytest.raises(eb.EtaError):
        eb.eta_fork_pages(64, 64, t, t, t.view(4, 1), t, t, t[:1], t, t, t)
