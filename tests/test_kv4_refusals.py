"""The index and the decode step of a 4-bit cache refuse on the host what they cannot do: no device is touched."""
import ctypes

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild


@pytest.fixture(scope="module")
def lib():
    ebuild.build()
    return eb.load()


ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)
DESC = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, block_size=64, t_cap=4096, nb_cap=64, k_stride_b=0, k_stride_h=0,
            k_stride_t=0, v_stride_b=0, v_stride_h=0, v_stride_t=0)
KV4 = dict(stride_b=64 * 2 * 9216, stride_h=64 * 9216, stride_j=9216, k_scale=1.0, v_scale=1.0)
PAGES = dict(block_table=256, table_stride=64, n_pages=10)


def _parts(kw):
    d, q4 = eb.CacheDesc(**{**DESC, **{k: v for k, v in kw.items() if k in DESC}}), eb.Kv4Desc(**{**KV4, **{k: v for k, v in kw.items() if k in KV4}})
    pg = eb.PageTable(**{**PAGES, **{k: v for k, v in kw.items() if k in PAGES}}) if kw.get("paged") else None
    ref = lambda x, name: None if kw.get(name, 0) is None or x is None else ctypes.byref(x)  # noqa: E731
    return ref(d, "desc"), ref(q4, "kv4"), ref(pg, "pages"), lambda name: kw.get(name, ONE)


COMMON = [(dict(desc=None), -1), (dict(kv4=None), -1), (dict(batch=0), -1), (dict(head_dim=32), -2), (dict(block_size=256), -2),
          (dict(n_q_heads=48), -2), (dict(nb_cap=8), -1), (dict(batch=600), -2), (dict(pool=None), -1), (dict(pool=ODD), -2),
          (dict(k_scale=0.0), -1), (dict(v_scale=float("nan")), -1), (dict(stride_j=9217), -2), (dict(stride_j=9200), -1), (dict(stride_h=16), -1),
          (dict(stride_b=16), -1), (dict(paged=True, n_pages=0), -1), (dict(paged=True, table_stride=63), -1),
          (dict(paged=True, block_table=None), -1), (dict(seq_lens=None), -1)]


@pytest.mark.parametrize("kw,code", COMMON + [(dict(musig=None), -1), (dict(mnorm=None), -1), (dict(flags=4), -1), (dict(musig=ODD), -2)])
def test_index(lib, kw, code):
    desc, kv4, pages, arg = _parts(kw)
    for call in (lib.eta_build_block_summaries_kv4, lib.eta_append_summary_kv4):
        assert call(desc, kv4, pages, arg("pool"), arg("seq_lens"), arg("musig"), arg("mnorm"), kw.get("flags", 0), None) == code


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(musig=None), -1), (dict(mnorm=None), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(sel=None), -1), (dict(tau=None), -1),
    (dict(const=ONE), -1), (dict(params=None), -1), (dict(rescue_window=0), -1), (dict(lwb=-1), -1), (dict(q=ODD), -2), (dict(out=ODD), -2),
    (dict(musig=ODD), -2), (dict(ws=None), -3), (dict(ws=ODD), -3), (dict(ws_bytes=64), -3)])
def test_decode(lib, kw, code):
    desc, kv4, pages, arg = _parts(kw)
    p = eb.DecodeParams(**{k: v for k, v in kw.items() if k in ("rescue_window", "lwb")}).c()
    params = None if kw.get("params", 0) is None else ctypes.byref(p)
    assert lib.eta_decode_kv4(desc, kv4, pages, params, arg("q"), arg("pool"), arg("seq_lens"), arg("musig"), arg("mnorm"), arg("tau"),
                              kw.get("const"), arg("out"), arg("sel"), None, None, arg("ws"), kw.get("ws_bytes", 1 << 30), None) == code


def test_workspace(lib):
    d = eb.CacheDesc(**DESC)
    n = eb.eta_kv4_workspace_bytes(d)
    assert n > 0 and n % 256 == 0
    sz = ctypes.c_size_t(0)
    assert lib.eta_kv4_workspace_bytes(None, ctypes.byref(sz)) == lib.eta_kv4_workspace_bytes(ctypes.byref(d), None) == -1
    with pytest.raises(eb.EtaError):
        eb.eta_kv4_workspace_bytes(eb.CacheDesc(**{**DESC, "head_dim": 96}))


def test_binding_refuses_host_tensors_and_other_structures(lib):
    pool = torch.zeros((2, 2, 3, 9216), dtype=torch.uint8)
    desc, kv4 = eb.kv4_cache_desc(pool, 8, 128, 64)
    with pytest.raises(eb.EtaError, match="pool must be a CUDA tensor"):
        eb.eta_build_block_summaries_kv4(desc, kv4, pool, None, None, None)
    with pytest.raises(eb.EtaError, match="pool must be"):
        eb.eta_append_summary_kv4(desc, kv4, None, None, None, None)
    with pytest.raises(TypeError):
        eb.eta_append_summary_kv4(desc, desc, pool, None, None, None)
    with pytest.raises(TypeError):
        eb.eta_decode_kv4(desc, None, eb.DecodeParams(), *[None] * 9, None)
    with pytest.raises(eb.EtaError, match="pool must be a CUDA tensor"):
        eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(), None, pool, *[None] * 7, None)
