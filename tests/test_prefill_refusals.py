"""Attention of a step's new tokens: what the entry point refuses, and how it shares out the work.  On the CPU, no device is touched."""
import ctypes
import random

import pytest

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild


@pytest.fixture(scope="module")
def lib():
    ebuild.build()
    return eb.load()


def _desc(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, block_size=64, t_cap=4096, nb_cap=64, k_stride_b=2 * 4096 * 128,
                k_stride_h=4096 * 128, k_stride_t=128, v_stride_b=2 * 4096 * 128, v_stride_h=4096 * 128, v_stride_t=128)
    base.update(kw)
    return eb.CacheDesc(**base)


ONE, NULL = ctypes.c_void_p(256), ctypes.c_void_p(None)


def _call(lib, **kw):
    a = dict(desc=_desc(), pages=None, flags=0, n_rows=10, q=ONE, row_start=ONE, seq_lens=ONE, granted=NULL, K=ONE, V=ONE, tau=ONE, const=NULL, out=ONE,
             ws=ONE, ws_bytes=1 << 40, params=True)
    a.update(kw)
    p = eb.DecodeParams(flags=a["flags"]).c()
    desc = ctypes.byref(a["desc"]) if a["desc"] is not None else None
    return lib.eta_prefill(desc, ctypes.byref(a["pages"]) if a["pages"] else None, ctypes.byref(p) if a["params"] else None, a["n_rows"],
                           a["q"], a["row_start"], a["seq_lens"], a["granted"], a["K"], a["V"], a["tau"], a["const"], a["out"], NULL, a["ws"],
                           a["ws_bytes"], NULL)


@pytest.mark.parametrize("kw,code", [
    (dict(desc=None), -1), (dict(desc=_desc(head_dim=96)), -2), (dict(desc=_desc(block_size=16)), -2), (dict(desc=_desc(n_q_heads=6)), -2),
    (dict(desc=_desc(n_q_heads=7)), -1), (dict(desc=_desc(batch=1025)), -2), (dict(desc=_desc(batch=0)), -1),
    (dict(desc=_desc(n_q_heads=2048, n_kv_heads=2048)), -2), (dict(desc=_desc(k_stride_t=100)), -2), (dict(desc=_desc(v_stride_t=64)), -1),
    (dict(params=False), -1), (dict(n_rows=-1), -1), (dict(n_rows=(1 << 30) + 1), -2), (dict(q=NULL), -1), (dict(out=NULL), -1), (dict(row_start=NULL), -1),
    (dict(seq_lens=NULL), -1), (dict(K=NULL), -1), (dict(V=NULL), -1), (dict(const=ONE), -1), (dict(tau=NULL), -1),
    (dict(q=ctypes.c_void_p(264)), -2), (dict(out=ctypes.c_void_p(258)), -2), (dict(K=ctypes.c_void_p(264)), -2), (dict(V=ctypes.c_void_p(264)), -2),
    (dict(ws=NULL), -3), (dict(ws=ctypes.c_void_p(128)), -3), (dict(ws_bytes=1 << 20), -3),
    (dict(pages=eb.PageTable(NULL, 64, 10)), -1), (dict(pages=eb.PageTable(ONE, 63, 10)), -1), (dict(pages=eb.PageTable(ONE, 64, 0)), -1),
])
def test_refused_before_any_launch(lib, kw, code):
    assert _call(lib, **kw) == code


def test_no_rows_is_nothing_to_do(lib):
    assert _call(lib, n_rows=0, q=NULL, out=NULL) == 0


def test_workspace_bytes(lib):
    n = eb.eta_prefill_workspace_bytes(_desc())
    assert n % 256 == 0 and n > 0
    # by the head's size only
    assert eb.eta_prefill_workspace_bytes(_desc(batch=64, t_cap=1 << 20)) == n
    assert eb.eta_prefill_workspace_bytes(_desc(head_dim=64)) < n
    size = ctypes.c_size_t(0)
    assert lib.eta_prefill_workspace_bytes(ctypes.byref(_desc()), None) == -1
    assert lib.eta_prefill_workspace_bytes(ctypes.byref(_desc(head_dim=32)), ctypes.byref(size)) == -2


def test_a_cpu_tensor_is_refused():
    import torch
    t = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(eb.EtaError):
        eb.eta_prefill(_desc(), eb.DecodeParams(flags=1), t, t, t, t, t, t, t)


def _shares(lib, heads, g_shift, d, ctas, n, lens):
    whole = ctypes.c_int(0)
    ints = ctypes.c_int32 * len(n)
    return lib.eta_selftest_prefill_shares(len(n), heads, g_shift, d, ctas, ints(*n), ints(*lens), ctypes.byref(whole)), whole.value


def test_every_tile_is_in_one_share(lib):
    rng = random.Random(0)
    ways = [0, 0]
    for _ in range(1500):
        n = [rng.choice([0, 1, 1, rng.randint(1, 300), int(2 ** rng.uniform(0, 12))]) for _ in range(rng.choice([1, 1, 2, 3, rng.randint(1, 150)]))]
        lens = [max(0, x + rng.choice([0, 0, rng.randint(0, 500), int(2 ** rng.uniform(0, 17)), -rng.randint(0, 50)])) for x in n]
        rc, whole = _shares(lib, rng.choice([1, 2, 3, 8]), rng.randint(0, 3), rng.choice([64, 128]), rng.choice([148, 148, 132, 160, 1, 7]), n, lens)
        assert rc == 0, (rc, n, lens)
        ways[whole] += 1
    assert min(ways) > 100


def test_long_sequences_keep_their_count(lib):
    assert _shares(lib, 8, 2, 128, 148, [1], [(1 << 31) - 1])[0] == 0
    assert _shares(lib, 8, 0, 128, 148, [100000, 3], [1 << 24, 1 << 30])[0] == 0
