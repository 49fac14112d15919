"""eta_plan_pages refuses on the host what it cannot do: no device is touched."""
import ctypes

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild


@pytest.fixture(scope="module")
def lib():
    ebuild.build()
    return eb.load()


ORDER = ("batch", "block_size", "t_cap", "new_lens", "release", "seq_lens", "seq_lens_out", "block_table", "table_stride", "free_pages",
         "n_free", "n_free_out", "n_pages", "n_rows", "slot_map", "positions", "row_start", "granted", "status", "stream")


def _call(lib, **kw):
    one = ctypes.c_void_p(256)                     # never dereferenced on the host
    args = dict(batch=2, block_size=64, t_cap=4096, new_lens=one, release=None, seq_lens=one, seq_lens_out=one, block_table=one,
                table_stride=64, free_pages=one, n_free=one, n_free_out=one, n_pages=128, n_rows=8, slot_map=one, positions=one,
                row_start=one, granted=one, status=None, stream=None)
    args.update(kw)
    return lib.eta_plan_pages(*(args[k] for k in ORDER))


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(batch=-3), -1), (dict(t_cap=0), -1), (dict(table_stride=0), -1), (dict(n_pages=0), -1),
    (dict(n_rows=-1), -1), (dict(block_size=48), -2), (dict(block_size=0), -2), (dict(t_cap=4097), -1), (dict(table_stride=63), -1),
    (dict(new_lens=None), -1), (dict(seq_lens=None), -1), (dict(seq_lens_out=None), -1), (dict(block_table=None), -1),
    (dict(free_pages=None), -1), (dict(n_free=None), -1), (dict(n_free_out=None), -1), (dict(row_start=None), -1),
    (dict(granted=None), -1), (dict(slot_map=None), -1), (dict(positions=None), -1), (dict(n_rows=(1 << 30) + 1), -2),
    (dict(slot_map=ctypes.c_void_p(260)), -2), (dict(n_pages=(1 << 30) + 1), -2), (dict(batch=(1 << 30) + 1), -2)])
def test_refusals(lib, kw, code):
    assert _call(lib, **kw) == code


def test_binding_refuses_host_tensors_and_what_is_missing(lib):
    i = torch.zeros(2, dtype=torch.int32)
    slots = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(eb.EtaError, match="new_lens must be a CUDA tensor"):
        eb.eta_plan_pages(64, 4096, i, i, i.view(1, 2), i, i, slots, i, i, i)
    with pytest.raises(eb.EtaError, match="new_lens must be a tensor"):
        eb.eta_plan_pages(64, 4096, None, i, i.view(1, 2), i, i, slots, i, i, i)
    with pytest.raises(OverflowError):
        eb.eta_plan_pages(64, 1 << 40, i, i, i.view(1, 2), i, i, slots, i, i, i)
