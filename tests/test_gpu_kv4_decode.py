"""eta_decode_kv4 against the oracle's decode step on the keys and values that the cache stands for (bf16 numbers at the tensors' scales used
here), from the same summaries and thresholds: masks equal outside the near-tie band, outputs within what fp32 arithmetic allows."""
import warnings

import numpy as np
import pytest
import torch

from oracle import eta_oracle as orc
from tests import kv4_reference as ref
from tests.helpers import bf16_bits_from_f64, bf16_values, compare_masks, heads_without_near_tie

pytestmark = pytest.mark.gpu


def case(seed, B, Hkv, G, d, b, lens, kscale=1.0, kg=1.0, vg=0.75, extra=0):
    """A cache, its index and a step's queries; lengths beyond `lens` hold garbage of the format (NaN scales among it)."""
    rng = np.random.default_rng(seed)
    nb = max(1, -(-max(lens) // b)) + extra
    K, V = (rng.standard_normal((B, Hkv, nb * b, d)) * s for s in (kscale, 1.0))
    blocks = ref.pack(K, V, b, kg, vg)
    K, V = ref.unpack(blocks, b, d, kg, vg)
    views = ref.split(blocks, b, d)
    for i, n in enumerate(lens):
        for x in views:
            y = x[i].reshape(Hkv, nb * b, -1)
            y[:, n:] = rng.integers(0, 256, y[:, n:].shape, np.uint8)
            x[i] = y.reshape(x[i].shape)
    blocks = np.concatenate([x.reshape(*x.shape[:-2], -1) for x in views], -1)
    q = bf16_bits_from_f64(rng.standard_normal((B, Hkv * G, d)))
    lens = np.asarray(lens, np.int32)
    c = orc.Cache(bf16_bits_from_f64(K), bf16_bits_from_f64(V), lens, b)
    assert np.array_equal(bf16_values(c.K), K) and np.array_equal(bf16_values(c.V), V)
    return dict(rng=rng, blocks=blocks, c=c, K=K, V=V, q=q, lens=lens, b=b, d=d, G=G, kg=kg, vg=vg)


def gpu(s, musig, mnorm, tau=None, const=None, paged=False, flags=0, q=None, status=True, **kw):
    from paper_2609_20888_b200 import binding as eb
    B, Hkv, nb, _ = s["blocks"].shape
    Hq = Hkv * s["G"]
    table = None
    blocks = s["blocks"]
    if paged:
        blocks, table = ref.scatter(blocks, np.random.default_rng(1))
        table = torch.from_numpy(table).cuda()
    pool = torch.from_numpy(blocks).cuda()
    desc, kv4 = eb.kv4_cache_desc(pool, Hq, s["d"], s["b"], batch=B, t_cap=nb * s["b"], k_scale=s["kg"], v_scale=s["vg"])
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    out = torch.full((B, Hq, s["d"]), float("nan"), device="cuda")
    sel = torch.full((B, Hkv, nb), 0xee, dtype=torch.uint8, device="cuda")
    stats, st = torch.zeros((B, Hkv), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    n = eb.eta_kv4_workspace_bytes(desc)
    ws = torch.full((n + 256,), 0xff, dtype=torch.uint8, device="cuda")
    ws = ws[-ws.data_ptr() % 256:][:n]
    ms = None if musig is None else dev(musig.view(np.int16)).view(torch.float16) if musig.dtype == np.uint16 else dev(musig)
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=flags, **kw), dev((s["q"] if q is None else q).view(np.int16)).view(torch.bfloat16), pool,
                      dev(s["lens"]), ms, dev(mnorm), dev(tau), dev(const), out, sel, ws, stats=stats, status=st,
                      pages=None if table is None else eb.page_table(table, len(blocks)))
    torch.cuda.synchronize()
    return out.cpu().numpy(), sel.cpu().numpy(), stats.cpu().numpy(), int(st.item())


def check(s, got, want, tau, beta, scale=None):
    out, sel, stats, _ = got
    B, Hkv, nb = sel.shape
    near = compare_masks(sel, want["sel"], want["bound"], tau, s["lens"], s["b"], s["G"], rescued=want["rescued"])
    keep = heads_without_near_tie(near, B, Hkv * s["G"])
    assert keep.mean() > 0.9
    tol = ref.output_bound(bf16_values(s["q"]), s["K"], s["V"], beta, 1 / np.sqrt(s["d"]) if scale is None else scale)
    err = np.abs(out - want["out"])[keep]
    assert err.max() <= tol, (err.max(), tol)
    assert np.array_equal(stats, (sel != 0).sum(2))


def _draw(seed):
    rng = np.random.default_rng(4000 + seed)
    d, b, G = int(rng.choice([64, 128])), int(rng.choice([32, 64, 128])), int(rng.choice([1, 2, 4, 8]))
    B, Hkv = int(rng.integers(1, 6)), int(rng.choice([1, 2, 3]))
    lens = []
    for _ in range(B):
        kind = rng.integers(0, 10)
        lens.append(int(rng.integers(1, b)) if kind == 0 else int(rng.integers(1, 4)) * b if kind == 1
                    else int(rng.integers(b, 96 * b if b == 32 else 30 * b)))
    return dict(seed=seed, B=B, Hkv=Hkv, G=G, d=d, b=b, lens=lens, kscale=float(rng.choice([0.3, 1.0, 3.0])), kg=float(rng.choice([1.0, 0.75, 0.5])),
                vg=float(rng.choice([1.0, 1.5])), extra=int(rng.choice([0, 0, 3]))), dict(
        quantile=float(rng.choice([0.0, 0.3, 0.6, 0.9, 0.98])), a=float(rng.choice([0.0, 0.0, 0.25, -0.5])), z=float(rng.choice([0.0, 0.5, 1.0, 2.5])),
        beta=float(rng.choice([0.0, 1.0, 5.0, 20.0])), lwb=int(rng.choice([0, 0, 1, 3])), rescue_window=int(rng.choice([1, 2, 128, 1 << 20])),
        ungate=bool(rng.integers(0, 2)), frozen=bool(rng.integers(0, 3) == 0), paged=bool(rng.integers(0, 2)))


@pytest.mark.parametrize("seed", range(40))
def test_random_configuration_matches_the_oracle(seed):
    kw, p = _draw(seed)
    s = case(**kw)
    B, Hq = kw["B"], kw["Hkv"] * kw["G"]
    musig, mnorm = orc.block_summaries(s["c"])
    bound = orc.score_dual(s["q"], musig, mnorm, s["lens"], s["b"], p["z"])
    with np.errstate(all="ignore"), warnings.catch_warnings():
        warnings.simplefilter("ignore")
        cut = np.nan_to_num(np.nanquantile(bound, p["quantile"], axis=2), nan=0.0) + p["a"] + 3e-4
    tau, const = cut.astype(np.float32), None
    if p["frozen"]:
        tau, const = None, np.median(cut, 0).astype(np.float32)
    used = np.broadcast_to(const, (B, Hq)) if p["frozen"] else tau
    how = {k: p[k] for k in ("z", "a", "beta", "lwb", "rescue_window")}
    want = orc.decode_step(s["q"], s["c"], musig, mnorm, tau=tau, head_const=const, ungate_last=p["ungate"], **how)
    got = gpu(s, musig, mnorm, tau, const, paged=p["paged"], flags=2 if p["ungate"] else 0, **how)
    assert got[3] == 0
    check(s, got, want, used.astype(np.float64) - p["a"], p["beta"])
    again = gpu(s, musig, mnorm, tau, const, paged=not p["paged"], flags=2 if p["ungate"] else 0, **how)
    assert all(np.array_equal(x, y) for x, y in zip(got, again))          # paged or not: the same bits


@pytest.mark.parametrize("d,b,G", [(64, 32, 8), (64, 64, 1), (64, 128, 4), (128, 32, 2), (128, 64, 8), (128, 128, 8), (128, 64, 4)])
def test_every_block_ungated(d, b, G):
    """ETA_FLAG_DENSE: softmax attention, without an index; lengths from one token on."""
    s = case(d + b + G, 6, 2, G, d, b, [1, b - 1, b, b + 1, 7 * b + 3, 21 * b])
    want = orc.dense_softmax_attention(s["q"], s["c"])
    got = gpu(s, None, None, tau=np.zeros((6, 2 * G), np.float32), flags=1)
    tol = ref.output_bound(bf16_values(s["q"]), s["K"], s["V"], 0.0, 1 / np.sqrt(d))
    assert np.abs(got[0] - want).max() <= tol
    assert np.array_equal(got[2], np.repeat((s["lens"] // b)[:, None], 2, 1)) and got[3] == 0


@pytest.mark.parametrize("power", [-100, -30, 40])
def test_queries_beyond_fp16(power):
    """Queries are scaled by a power of two per head: magnitudes that fp16 cannot hold attend like any others."""
    s = case(5, 2, 2, 4, 128, 64, [500, 64 * 9])
    s["q"] = bf16_bits_from_f64(bf16_values(s["q"]) * 2.0 ** power)
    want = orc.dense_softmax_attention(s["q"], s["c"], scale=2.0 ** -power / 11)
    got = gpu(s, None, None, tau=np.zeros((2, 8), np.float32), flags=1, scale=2.0 ** -power / 11)
    tol = ref.output_bound(bf16_values(s["q"]) * 2.0 ** -power, s["K"], s["V"], 0.0, 1 / 11)
    assert np.abs(got[0] - want).max() <= tol


def test_empty_and_overlong_sequences():
    s = case(9, 3, 1, 2, 64, 32, [0, 96, 40], extra=0)
    musig, mnorm = orc.block_summaries(s["c"])
    tau = np.full((3, 2), -1e30, np.float32)
    out, sel, stats, status = gpu(s, musig, mnorm, tau)
    want = orc.decode_step(s["q"], s["c"], musig, mnorm, tau=tau)
    assert status == 4 and not out[0].any() and not sel[0].any() and stats.tolist() == [[0], [3], [1]]
    assert np.abs(out - want["out"]).max() <= ref.output_bound(bf16_values(s["q"]), s["K"], s["V"], 5.0, 0.125)
    s["lens"] = np.array([0, 1000, 40], np.int32)
    again = gpu(s, musig, mnorm, tau)
    assert again[3] == 4 | 2 and np.array_equal(again[0][1:], out[1:])


@pytest.mark.parametrize("d,b,G", [(128, 64, 4), (64, 32, 8), (128, 128, 2)])
def test_a_nan_reaches_the_heads_that_attend_its_block_and_no_others(d, b, G):
    s = case(11, 1, 1, G, d, b, [12 * b])
    musig, mnorm = orc.block_summaries(s["c"])
    bound = orc.score_dual(s["q"], musig, mnorm, s["lens"], b, 1.0)
    tau = np.median(bound, 2).astype(np.float32) + np.float32(3e-4)
    tau[0, 0] = -100                                          # head 0 attends everything
    clean = gpu(s, musig, mnorm, tau)
    sel = clean[1][0, 0]
    j = int(np.argmax([(x & 1) * (int(x) != (1 << G) - 1) * bin(int(x)).count("1") for x in sel]))
    on = [(int(sel[j]) >> g) & 1 for g in range(G)]
    assert on[0] and not all(on)
    c, e = b * d // 2, b * d // 16
    s["blocks"][0, 0, j, 2 * c + e + (d // 16) * 5 + 2] = 0x7f      # the value of token 5, channels 32 .. 47
    got = gpu(s, musig, mnorm, tau)
    assert np.array_equal(got[1], clean[1])
    for g in range(G):
        if on[g]:
            nan = np.isnan(got[0][0, g])
            assert nan[32:48].all() and nan.sum() == 16 and np.array_equal(got[0][0, g][~nan], clean[0][0, g][~nan])
        else:
            assert np.array_equal(got[0][0, g], clean[0][0, g])
    s["blocks"][0, 0, j, c + (d // 16) * 5 + 1] = 0xff              # and its key
    got = gpu(s, musig, mnorm, tau)
    for g in range(G):
        assert np.isnan(got[0][0, g]).all() if on[g] else np.array_equal(got[0][0, g], clean[0][0, g])


def test_a_query_that_is_no_number():
    s = case(12, 2, 1, 4, 128, 64, [300, 64])
    s["q"][1, 2, 7] = 0x7fc0
    got = gpu(s, None, None, tau=np.zeros((2, 4), np.float32), flags=1)[0]
    nan = np.isnan(got)
    assert nan[1, 2].all() and nan.sum() == 128


def test_packed_summaries_and_many_rows():
    """128 sequences of very different lengths, eight heads, the packed index."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(1, 1500, 128)]
    s = case(13, 128, 2, 8, 64, 32, lens)
    m8, mnorm = orc.block_summaries_sigma8(s["c"])
    musig = orc.unpack_sigma8(m8)
    bound = orc.score_dual(s["q"], musig, mnorm, s["lens"], 32, 1.0)
    with np.errstate(all="ignore"), warnings.catch_warnings():
        warnings.simplefilter("ignore")
        tau = (np.nan_to_num(np.nanquantile(bound, 0.7, axis=2)) + 3e-4).astype(np.float32)
    want = orc.decode_step(s["q"], s["c"], musig, mnorm, tau=tau)
    check(s, gpu(s, m8, mnorm, tau, flags=4), want, tau.astype(np.float64), 5.0)


@pytest.mark.parametrize("d,b,G,longest", [(128, 64, 4, 9000), (128, 32, 8, 9000), (64, 64, 8, 18000), (64, 128, 2, 18000)])
def test_long_pieces_with_growing_scores(d, b, G, longest):
    """160 rows, one or two to a CTA, whose running sums are put together many times over while their maxima still grow."""
    from paper_2609_20888_b200 import binding as eb
    B, Hkv, nb = 20, 8, -(-longest // b)
    g = torch.Generator(device="cuda").manual_seed(d + b)
    pool = torch.randint(0, 256, (B, Hkv, nb, eb.kv4_block_bytes(b, d)), dtype=torch.uint8, device="cuda", generator=g)
    k0, v0, sc = b * d // 2, b * d // 2 + b * d // 16, b * d // 16
    step = (torch.arange(nb * b, device="cuda") * 3 // (nb * b)).to(torch.uint8).reshape(nb, b, 1).expand(nb, b, d // 16).reshape(nb, sc)
    pool[..., k0:k0 + sc] = 0x20 + 8 * step                # 2^-3, 2^-2 and 2^-1
    pool[..., v0 + b * d // 2:] = 0x30
    lens = torch.randint(longest // 2, longest + 1, (B,), dtype=torch.int32, device="cuda", generator=g)
    q = torch.randn((B, Hkv * G, d), device="cuda", generator=g).to(torch.bfloat16)
    desc, kv4 = eb.kv4_cache_desc(pool, Hkv * G, d, b, batch=B, t_cap=nb * b)
    out, st = torch.empty((B, Hkv * G, d), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    sel = torch.empty((B, Hkv, nb), dtype=torch.uint8, device="cuda")
    ws = torch.empty(eb.eta_kv4_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), q, pool, lens, None, None, torch.zeros((B, Hkv * G), device="cuda"), None,
                      out, sel, ws, status=st)
    K, V = (torch.empty((B, Hkv, nb * b, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eb.eta_unpack_kv4(desc, kv4, pool, K, V)
    assert st.item() == 0
    for i in range(B):
        n = int(lens[i])
        x, y = K[i, :, :n].double(), V[i, :, :n].double()
        want = torch.softmax(q[i].double().reshape(Hkv, G, d) @ x.mT / d ** 0.5, -1) @ y
        # fp32 arithmetic, and an MMA's sum that is cut off 2^-22 below its own size, at most 80 times before it is put away
        tol = ref.output_bound(q[i].double().cpu().numpy(), x.cpu().numpy(), y.cpu().numpy(), 0.0, d ** -0.5) + 80 * 2.0 ** -22 * float(y.abs().max())
        assert float((out[i].reshape(Hkv, G, d).double() - want).abs().max()) <= tol


def test_offsets_past_32_bits():
    """Pages more than 2^31 bytes apart: written by the token call, indexed, attended."""
    from paper_2609_20888_b200 import binding as eb
    d, b, Hkv, G, n = 128, 64, 2, 4, 150
    size, apart = eb.kv4_block_bytes(b, d), (1 << 31) + 4096
    raw = torch.zeros(3 * apart + 2 * size, dtype=torch.uint8, device="cuda")
    far = raw.as_strided((4, Hkv, size), (apart, size, 1))
    near = torch.zeros((4, Hkv, size), dtype=torch.uint8, device="cuda")
    g = torch.Generator().manual_seed(0)
    qkv = torch.randn((n, Hkv * (G + 2), d), generator=g).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :Hkv * G], qkv[:, Hkv * G:Hkv * (G + 1)], qkv[:, Hkv * (G + 1):]
    table = torch.tensor([[3, 1, 2]], dtype=torch.int32, device="cuda")
    t = torch.arange(n, device="cuda")
    slots = table[0, t // b].long() * b + t % b
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    res = []
    for pool in (far, near):
        desc, kv4 = eb.kv4_cache_desc(pool, Hkv * G, d, b, batch=1, t_cap=3 * b)
        q_out = torch.empty((n, Hkv * G, d), dtype=torch.bfloat16, device="cuda")
        eb.eta_append_tokens_kv4(desc, kv4, q, k, v, slots, None, q_out, pool)
        musig, mnorm = eb.alloc_summaries(desc, "cuda")
        pages = eb.page_table(table, 4)
        eb.eta_build_block_summaries_kv4(desc, kv4, pool, lens, musig, mnorm, pages=pages)
        ws = torch.empty(eb.eta_kv4_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        out, sel = torch.empty((1, Hkv * G, d), device="cuda"), torch.empty((1, Hkv, 3), dtype=torch.uint8, device="cuda")
        eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(), q_out[-1:], pool, lens, musig, mnorm, torch.zeros((1, Hkv * G), device="cuda"), None, out, sel,
                          ws, pages=pages)
        K, V = (torch.empty((4, Hkv, b, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        eb.eta_unpack_kv4(desc, kv4, pool, K, V)
        res.append((q_out, musig, mnorm, out, sel, K, V))
    for x, y in zip(*res):
        assert torch.equal(x, y)
    assert res[0][3].isfinite().all() and res[0][3].any()
