"""Tensor scales as a calibration gives them, largest magnitude / (6 * 448), with all of fp32's bits: the bytes that are written, what they read back as, their
index and attention over them."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def calibrated(x):
    return float(np.float32(np.abs(x).max()) / np.float32(2688))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("norm,rotary,interleaved", [(True, 64, False), (True, 32, True), (False, 64, True), (False, 0, False), (True, 0, False)])
@pytest.mark.parametrize("which", ["both", "keys", "values"])
def test_bytes_written(dtype, norm, rotary, interleaved, which):
    from paper_2609_20888_b200 import binding as eb
    rows, heads, d, block = 96, 5, 64, 32
    rng = np.random.default_rng(31 * norm + rotary)
    x = rng.standard_normal((2, rows, heads, d)) * (1 + 3 * rng.random((heads, d)))
    k, v = (torch.from_numpy(y).to(DT[dtype]).cuda() for y in x)
    k64, v64 = (t.double().cpu().numpy() for t in (k, v))
    w = (rng.random(d) + 0.5).astype(np.float32) if norm else None
    inv = 10000.0 ** -(np.arange(rotary // 2) / max(1, rotary // 2))
    pos = rng.integers(0, 1 << 20, rows)
    y = ref.norm(k64, w, 1e-6)
    y = ref.rotate(y, pos, inv, interleaved) if rotary else y
    kg, vg = (calibrated(y) if which != "values" else 1.0), (calibrated(v64) if which != "keys" else 0.5)
    pool = torch.zeros((rows // block, heads, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
    desc, kv4 = eb.kv4_cache_desc(pool, heads, d, block, batch=1, t_cap=block, k_scale=kg, v_scale=vg)
    q_out = torch.empty((rows, heads, d), dtype=torch.bfloat16, device="cuda")
    eb.eta_append_tokens_kv4(desc, kv4, k, k, v, torch.arange(rows, device="cuda"), torch.from_numpy(pos.astype(np.int32)).cuda(), q_out, pool,
                             inv_freq=torch.from_numpy(inv).cuda() if rotary else None, k_weight=None if w is None else torch.from_numpy(w).cuda(),
                             interleaved=interleaved)
    got = [z.transpose(0, 2, 1, 3).reshape(rows, heads, -1) for z in ref.split(pool.cpu().numpy(), block, d)]
    for at, want, g in ((0, y, kg), (2, v64, vg)):
        codes, scales = ref.encode(want, g)
        assert np.array_equal(got[at + 1], scales) and np.array_equal(got[at], codes)
    K, V = (torch.zeros((rows // block, heads, block, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eb.eta_unpack_kv4(desc, kv4, pool, K, V)
    for t, at, g in ((K, 0, kg), (V, 2, vg)):
        want = ref.decode(got[at], got[at + 1], g)
        back = t.double().cpu().numpy().transpose(0, 2, 1, 3).reshape(rows, heads, d)
        # scale * g and its product with a code in fp32, then bf16
        assert (np.abs(back - want) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(want)).all()


@pytest.mark.parametrize("G,d,b", [(4, 128, 64), (8, 64, 32)])
def test_index_and_dense_attention(G, d, b):
    from paper_2609_20888_b200 import binding as eb
    rng = np.random.default_rng(8)
    B, Hkv, nb = 2, 2, 5
    K, V = (rng.standard_normal((B, Hkv, nb * b, d)) * s for s in (1.3, 0.7))
    kg, vg = calibrated(K), calibrated(V)
    blocks = ref.pack(K, V, b, kg, vg)
    K, V = ref.unpack(blocks, b, d, kg, vg)
    pool = torch.from_numpy(blocks).cuda()
    desc, kv4 = eb.kv4_cache_desc(pool, Hkv * G, d, b, k_scale=kg, v_scale=vg)
    lens = np.array([nb * b, 3 * b + 7], np.int32)
    lens_d = torch.from_numpy(lens).cuda()
    musig, mnorm = eb.alloc_summaries(desc, torch.device("cuda"))
    eb.eta_build_block_summaries_kv4(desc, kv4, pool, lens_d, musig, mnorm)
    ms, mn = musig.double().cpu().numpy().reshape(B, Hkv, nb, 2, d), mnorm.double().cpu().numpy().reshape(B, Hkv, nb)
    for i in range(B):
        n = lens[i] // b
        k = K[i].reshape(Hkv, nb, b, d)[:, :n]
        size = np.abs(k).max(2)
        # fp32 sums of at most 128 numbers (2^-20 of the largest is ample), one rounding to fp16
        assert (np.abs(ms[i, :, :n, 0] - k.mean(2)) <= 2.0 ** -11 * np.abs(k.mean(2)) + 2.0 ** -20 * size + 2.0 ** -25).all()
        # of the deviation: its square is off by at most 2^-20 of size^2, the root by that over the deviation
        sd = k.std(2)
        assert (np.abs(ms[i, :, :n, 1] - sd) <= 2.0 ** -11 * sd + 2.0 ** -20 * size ** 2 / sd + 2.0 ** -25).all()
        norms = np.sqrt((k ** 2).sum(-1)).max(2)
        assert (np.abs(mn[i, :, :n] - norms) <= 2.0 ** -19 * norms).all()
    q = torch.from_numpy(rng.standard_normal((B, Hkv * G, d))).to(torch.bfloat16).cuda()
    out = torch.empty((B, Hkv * G, d), device="cuda")
    sel = torch.zeros((B, Hkv, nb), dtype=torch.uint8, device="cuda")
    n = eb.eta_kv4_workspace_bytes(desc)
    raw = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), q, pool, lens_d, None, None,
                      torch.zeros((B, Hkv * G), device="cuda"), None, out, sel,
                      raw[-raw.data_ptr() % 256:][:n], status=status)
    assert status.item() == 0
    q64, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    scale = 1 / np.sqrt(d)
    for i in range(B):
        for h in range(Hkv * G):
            k, v = K[i, h // G, :lens[i]], V[i, h // G, :lens[i]]
            s = k @ q64[i, h] * scale
            p = np.exp(s - s.max())
            assert np.abs(got[i, h] - (p / p.sum()) @ v).max() <= ref.output_bound(q64[i, h][None], k, v, 0.0, scale)
