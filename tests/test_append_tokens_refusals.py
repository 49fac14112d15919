"""eta_append_tokens, its 4-bit form and eta_unpack_kv4 refuse on the host what they cannot do: no device is touched."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from paper_2609_20888_b200 import build as ebuild
from tests import kv4_reference as ref


@pytest.fixture(scope="module")
def lib():
    ebuild.build()
    return eb.load()


ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)
DESC = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, block_size=64, t_cap=4096, nb_cap=64, k_stride_b=1 << 20, k_stride_h=1 << 19,
            k_stride_t=128, v_stride_b=1 << 20, v_stride_h=1 << 19, v_stride_t=128)
TOK = dict(n_rows=4, type=0, rotary_dim=128, flags=0, q_stride_r=1536, q_stride_h=128, k_stride_r=1536, k_stride_h=128, v_stride_r=1536,
           v_stride_h=128, eps=1e-6)
KV4 = dict(stride_b=64 * 2 * 9216, stride_h=64 * 9216, stride_j=9216, k_scale=1.0, v_scale=1.0)
ARGS = dict(q=ONE, k=ONE, v=ONE, q_weight=ONE, k_weight=ONE, inv_freq=ONE, positions=ONE, slot_map=ONE, n_pages=0, q_out=ONE, K=ONE, V=ONE)


def _call(lib, four, kw):
    part = lambda base: {**base, **{k: v for k, v in kw.items() if k in base}}  # noqa: E731
    d, t, a = eb.CacheDesc(**part(DESC)), eb.TokensDesc(**part(TOK)), part(ARGS)
    desc = None if kw.get("desc", 0) is None else ctypes.byref(d)
    tok = None if kw.get("tok", 0) is None else ctypes.byref(t)
    first = [a[k] for k in ("q", "k", "v", "q_weight", "k_weight", "inv_freq", "positions", "slot_map", "n_pages", "q_out")]
    if four:
        q4 = None if kw.get("kv4", 0) is None else ctypes.byref(eb.Kv4Desc(**part(KV4)))
        return lib.eta_append_tokens_kv4(desc, q4, tok, *first, a["K"], None, None)
    return lib.eta_append_tokens(desc, tok, *first, a["K"], a["V"], None, None)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(desc=None), -1), (dict(tok=None), -1), (dict(batch=0), -1), (dict(head_dim=96), -2), (dict(n_q_heads=6), -2), (dict(n_q_heads=7), -1),
    (dict(block_size=16), -2), (dict(n_rows=-1), -1), (dict(type=3), -1), (dict(type=-1), -1), (dict(flags=2), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(rotary_dim=-16), -1), (dict(rotary_dim=144), -1), (dict(rotary_dim=24), -2), (dict(n_pages=-1), -1),
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(slot_map=None), -1), (dict(q_out=None), -1), (dict(K=None), -1),
    (dict(inv_freq=None), -1), (dict(positions=None), -1), (dict(q_stride_r=1540), -2), (dict(k_stride_h=4), -2), (dict(v_stride_r=12), -2),
    (dict(type=2, q_stride_r=1538), -2), (dict(q=ODD), -2), (dict(k=ODD), -2), (dict(v=ODD), -2), (dict(q_out=ODD), -2), (dict(K=ODD), -2),
    (dict(q_weight=ODD), -2), (dict(k_weight=ODD), -2), (dict(slot_map=ctypes.c_void_p(260)), -2), (dict(positions=ctypes.c_void_p(258)), -2),
    (dict(n_rows=0), 0)])
def test_refusals(lib, four, kw, code):
    assert _call(lib, four, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(kv4=None), -1), (dict(k_scale=0.0), -1), (dict(v_scale=-1.0), -1), (dict(k_scale=float("inf")), -1), (dict(v_scale=float("nan")), -1),
    (dict(stride_b=9215), -2), (dict(stride_h=9224), -2), (dict(stride_j=9200 + 8), -2), (dict(stride_j=9200), -1), (dict(stride_h=4608), -1)])
def test_refusals_of_the_4_bit_cache(lib, kw, code):
    assert _call(lib, True, kw) == code


def test_unpack_and_block_bytes(lib):
    d, q4 = eb.CacheDesc(**DESC), eb.Kv4Desc(**KV4)
    call = lambda d=d, q4=q4, pool=ONE, n=0, K=ONE, V=ONE: lib.eta_unpack_kv4(  # noqa: E731
        None if d is None else ctypes.byref(d), None if q4 is None else ctypes.byref(q4), pool, n, K, V, None)
    assert call(d=None) == call(q4=None) == call(pool=None) == call(K=None) == call(V=None) == call(n=-1) == -1
    assert call(K=ODD) == call(pool=ODD) == call(d=eb.CacheDesc(**{**DESC, "k_stride_t": 132})) == -2
    assert [eb.kv4_block_bytes(b, h) for b in (32, 64, 128) for h in (64, 128)] == [2 * b * (h // 2 + h // 16) for b in (32, 64, 128) for h in (64, 128)]
    assert eb.kv4_block_bytes(48, 64) == eb.kv4_block_bytes(64, 96) == 0


def test_descriptor_of_a_pool(lib):
    pool = torch.zeros((3, 2, 5, 4608), dtype=torch.uint8)
    desc, kv4 = eb.kv4_cache_desc(pool, 4, 64, 64, k_scale=0.5)
    assert (desc.batch, desc.n_kv_heads, desc.t_cap, desc.nb_cap) == (3, 2, 320, 5)
    assert (kv4.stride_b, kv4.stride_h, kv4.stride_j, kv4.k_scale, kv4.v_scale) == (2 * 5 * 4608, 5 * 4608, 4608, 0.5, 1.0)
    for bad in (dict(batch=4), dict(t_cap=321)):
        with pytest.raises(eb.EtaError):
            eb.kv4_cache_desc(pool, 4, 64, 64, **bad)
    for bad in (pool[0], pool.float(), pool[..., ::2], pool[..., :4592], pool[0, 0]):
        with pytest.raises(eb.EtaError):
            eb.kv4_cache_desc(bad, 4, 64, 64)


def test_binding_refuses_host_tensors(lib):
    q, k = torch.zeros((1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    K = torch.zeros((1, 2, 64, 64), dtype=torch.bfloat16)
    with pytest.raises(eb.EtaError, match="q must be a CUDA tensor"):
        eb.eta_append_tokens(eb.cache_desc(K, K, 4, 64), q, k, k, torch.zeros(1, dtype=torch.int64), None, q, K, K)
    with pytest.raises(TypeError):
        eb.eta_append_tokens(eb.cache_desc(K, K, 4, 64), None, k, k, torch.zeros(1, dtype=torch.int64), None, q, K, K)


def test_the_reference_of_the_format():
    """The definition that the GPU tests compare with, against torch's 8-bit type and by hand."""
    codes = torch.arange(127, dtype=torch.uint8)
    assert np.array_equal(ref.E4M3, codes.view(torch.float8_e4m3fn).double().numpy())
    x = np.zeros(32)
    x[:8] = [6, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5]           # ties, all to the even code
    x[16:20] = [12, 0.5, -0.51, 1.49]
    c, s = ref.encode(x, 1.0)
    assert s.tolist() == [0x38, 0x40]                           # 1 and 2
    assert ref.decode(c, s, 1.0)[:8].tolist() == [6, 0, 1, 1, 2, 2, 4, -4]
    assert ref.decode(c, s, 1.0)[16:20].tolist() == [12, 0, -1, 1]
    rng = np.random.default_rng(0)
    v = rng.standard_normal((50, 64))
    err = np.abs(ref.decode(*ref.encode(v, 0.75), 0.75) - v).reshape(50, 4, 16)
    top = np.abs(v).reshape(50, 4, 16).max(-1, keepdims=True)
    assert (err <= top * (1 / 6 + 1 / 16)).all()                # half the widest step (2 of 6), and the scale's rounding
