"""eta_append_tokens and eta_append_tokens_kv4 against their definition in 64 bits.

bf16 results: one rounding, off by at most 2^-8 of the value, after fp32 arithmetic that is off by at most 2^-19 of the pair's size (norm: a
sum of at most 128 squares in a tree of eights and four shuffles, a square root, two products, 2^-20; an angle reduced in 64 bits and rounded
to 32, and its sine and cosine, 2^-22; products and their sum, 2^-23).  4-bit results: bytes, equal."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def inputs(rows, hq, hkv, d, dtype, seed, layout="fused"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, hq + 2 * hkv, d), generator=g)
    x[:, hq:hq + hkv] *= 1 + 3 * torch.rand((hkv, d), generator=g)
    x = x.to(DT[dtype])
    if layout == "fused":
        x = x.cuda()
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    parts = [x[:, a:b].cuda() for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]
    # heads outermost, rows padded
    return [torch.nn.functional.pad(p.transpose(0, 1).contiguous(), (0, 16))[..., :d].transpose(0, 1) for p in parts]


def expected(q, k, v, pos, wq, wk, inv, interleaved, eps=1e-6):
    """fp64 queries and keys, and how large the pairs are that they were turned from."""
    n64 = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    out = []
    for x, w in ((q, wq), (k, wk)):
        y = ref.norm(n64(x), n64(w), eps)
        size = np.abs(y)
        if inv is not None and len(inv):
            n = 2 * len(inv)
            a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
            both = size[..., a] + size[..., b]
            size = size.copy()
            size[..., a], size[..., b] = both, both
            y = ref.rotate(y, pos.cpu().numpy(), n64(inv), interleaved)
        out += [y, size]
    return (*out, n64(v))


def close(got, want, size):
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + 2.0 ** -19 * size) + 2.0 ** -19 * size + 1e-38).all()


CASES = [  # rows, hq, hkv, d, dtype, norm, rotary, interleaved, block, paged, layout
    (1, 8, 8, 64, "bf16", True, 64, False, 32, True, "fused"),
    (1, 1, 1, 128, "fp32", True, 128, False, 64, False, "fused"),
    (7, 32, 8, 128, "bf16", True, 128, False, 64, True, "fused"),
    (33, 4, 1, 64, "fp16", True, 32, True, 128, True, "split"),
    (64, 16, 2, 128, "bf16", False, 64, False, 32, False, "split"),
    (129, 6, 3, 64, "fp32", True, 16, False, 64, True, "fused"),
    (300, 3, 3, 128, "fp16", False, 0, False, 64, False, "fused"),
    (515, 24, 3, 64, "bf16", True, 64, True, 32, False, "fused"),
    (2500, 10, 5, 128, "bf16", True, 112, False, 64, True, "fused"),
]


def _setup(case, seed):
    rows, hq, hkv, d, dtype, norm, rotary, interleaved, block, paged, layout = case
    g = torch.Generator().manual_seed(seed)
    q, k, v = inputs(rows, hq, hkv, d, dtype, seed, layout)
    pos = torch.randint(0, 1 << 20, (rows,), generator=g).int().cuda()
    wq, wk = (torch.rand((2, d), generator=g) + 0.5).cuda() if norm else (None, None)
    inv = (10000.0 ** -(torch.arange(rotary // 2, dtype=torch.float64) / max(1, rotary // 2))).cuda() if rotary else None
    pages = 2 + (rows + block - 1) // block
    t_cap = 3 * block - 7 if not paged else None
    n = pages * block if paged else -(-rows * 2 // t_cap) * t_cap
    slots = torch.randperm(n, generator=g)[:rows]
    slots[::5] = -1 - slots[::5]                                   # skipped rows
    if rows == 1:
        slots[0] = n - 1
    return q, k, v, pos, wq, wk, inv, slots.cuda(), n, pages, t_cap, interleaved, hq, hkv, d, block, paged


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_bf16_cache(case):
    from paper_2609_20888_b200 import binding as eb
    q, k, v, pos, wq, wk, inv, slots, n, pages, t_cap, interleaved, hq, hkv, d, block, paged = _setup(case, 11)
    per = block if paged else t_cap
    # token-major pages in half of the cases
    shape = (n // per, per, hkv, d) if case[0] % 2 else (n // per, hkv, per, d)
    K, V = (torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if case[0] % 2:
        K, V = K.transpose(1, 2), V.transpose(1, 2)
    desc = eb.paged_cache_desc(K, V, 3, hq, t_cap=4 * block) if paged else eb.cache_desc(K, V, hq, block)
    q_out = torch.full((len(slots), hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eb.eta_append_tokens(desc, q, k, v, slots, pos, q_out, K, V, inv_freq=inv, q_weight=wq, k_weight=wk, interleaved=interleaved, paged=paged,
                         status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    yq, sq, yk, sk, yv = expected(q, k, v, pos, wq, wk, inv, interleaved)
    live = (slots >= 0).cpu().numpy()
    close(q_out[torch.from_numpy(live).cuda()], yq[live], sq[live])
    assert (q_out[torch.from_numpy(~live).cuda()] == 5).all()
    at = slots[slots >= 0]
    flat = lambda X: X.transpose(1, 2).reshape(n, hkv, d)  # noqa: E731
    close(flat(K)[at], yk[live], sk[live])
    assert torch.equal(flat(V)[at], v[torch.from_numpy(live).cuda()].to(torch.bfloat16))
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (flat(K)[rest] == 7).all() and (flat(V)[rest] == 7).all()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("kg,vg", [(1.0, 0.75)])
def test_kv4_cache_and_back(case, kg, vg):
    from paper_2609_20888_b200 import binding as eb
    q, k, v, pos, wq, wk, inv, slots, n, pages, t_cap, interleaved, hq, hkv, d, block, paged = _setup(case, 12)
    size = eb.kv4_block_bytes(block, d)
    pad = 32 * (case[0] % 2)                                     # blocks further apart than they are long
    if paged:
        raw = torch.full((pages, hkv, size + pad), 0x5a, dtype=torch.uint8, device="cuda")
        desc, kv4 = eb.kv4_cache_desc(raw[..., :size], hq, d, block, batch=3, t_cap=4 * block, k_scale=kg, v_scale=vg)
    else:
        raw = torch.full((n // t_cap, hkv, 3, size + pad), 0x5a, dtype=torch.uint8, device="cuda")
        desc, kv4 = eb.kv4_cache_desc(raw[..., :size], hq, d, block, t_cap=t_cap, k_scale=kg, v_scale=vg)
    pool = raw[..., :size]
    before = pool.cpu().numpy().copy()
    q_out = torch.full((len(slots), hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
    eb.eta_append_tokens_kv4(desc, kv4, q, k, v, slots, pos, q_out, pool, inv_freq=inv, q_weight=wq, k_weight=wk, interleaved=interleaved)
    torch.cuda.synchronize()
    yq, sq, yk, _, yv = expected(q, k, v, pos, wq, wk, inv, interleaved)
    live = (slots >= 0).cpu().numpy()
    close(q_out[torch.from_numpy(live).cuda()], yq[live], sq[live])
    at = slots.cpu().numpy()[live]
    want = before.copy()
    kc, ks, vc, vs = ref.split(want, block, d)
    if paged:
        put = lambda x, y: x.__setitem__((at // block, slice(None), at % block), y)  # noqa: E731
    else:
        put = lambda x, y: x.__setitem__((at // t_cap, slice(None), at % t_cap // block, at % t_cap % block), y)  # noqa: E731
    for x, g, codes, scales in ((yk[live], kg, kc, ks), (yv[live], vg, vc, vs)):
        c, s = ref.encode(x, g)
        put(codes, c)
        put(scales, s)
    want = np.concatenate([x.reshape(*x.shape[:-2], -1) for x in (kc, ks, vc, vs)], -1)
    got = pool.cpu().numpy()
    assert np.array_equal(got, want)
    assert (raw[..., size:] == 0x5a).all()
    # and read back: every token of the cache, in both orders of axes
    per = block if paged else t_cap
    K = torch.full((raw.shape[0], hkv, per, d), 3.0, dtype=torch.bfloat16, device="cuda")
    V = torch.full((raw.shape[0], per, hkv, d), 3.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    eb.eta_unpack_kv4(desc, kv4, pool, K, V)
    torch.cuda.synchronize()
    blocks = got if not paged else got[:, :, None]
    wk64, wv64 = (x[:, :, :per] for x in ref.unpack(blocks, block, d, kg, vg))
    # one rounding to bf16 at most; exact where the tensor's scale is a power of two
    assert np.array_equal(K.double().cpu().numpy(), wk64, equal_nan=True)
    gv = V.double().cpu().numpy()
    assert (np.abs(gv - wv64) <= 2.0 ** -8 * np.abs(wv64)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_kv4_ties_zeros_infinities_and_nans(dtype):
    """Values as they are (no norm, no rotation): every border between two codes and two scales, and what is no number."""
    from paper_2609_20888_b200 import binding as eb
    d, hkv, block = 64, 2, 32
    rng = np.random.default_rng(5)
    x = rng.standard_normal((32, hkv, d))
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -6])
    for r in range(8):
        x[r, :, 16:32] = mids * 2.0 ** (r - 5)                    # a border each, at scales that are powers of two
        x[r, :, :16] = rng.integers(-1, 2, 16) * 0.01
        x[r, 0, 0] = 6 * (1 + (2 * r + 1) / 16) * 2.0 ** (r - 4)   # the scale lies between two
    x[8] = 0
    x[9, :, :16] = -0.0
    x[10, 0, 3], x[10, 1, 20] = np.inf, -np.inf
    x[11, 0, 5], x[11, 1, 63] = np.nan, -np.nan
    x[12, :, :16] = 6 * 2.0 ** -10                                # the scale is half the smallest: to zero
    x[13, :, :16] = 6.1 * 2.0 ** -10                              # and just above: the smallest
    x[14, :, :16] = 60000                                         # beyond the largest
    t = torch.from_numpy(x).to(DT[dtype]).cuda()
    pool = torch.zeros((1, hkv, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
    desc, kv4 = eb.kv4_cache_desc(pool, hkv, d, block, batch=1, t_cap=block)
    q_out = torch.empty((32, hkv, d), dtype=torch.bfloat16, device="cuda")
    eb.eta_append_tokens_kv4(desc, kv4, t, t, t, torch.arange(32, device="cuda"), None, q_out, pool)
    got = ref.split(pool.cpu().numpy(), block, d)
    c, s = ref.encode(t.double().cpu().numpy(), 1.0)
    for k in (0, 2):
        assert np.array_equal(got[k][0], c.transpose(1, 0, 2)) and np.array_equal(got[k + 1][0], s.transpose(1, 0, 2))
    K, V = (torch.empty((1, hkv, block, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eb.eta_unpack_kv4(desc, kv4, pool, K, V)
    assert torch.equal(K.isnan(), V.isnan()) and K.isnan().sum() == 32 and not K.isinf().any()
    assert np.array_equal(K[0].double().cpu().numpy(), ref.decode(c, s, 1.0).transpose(1, 0, 2), equal_nan=True)


@pytest.mark.parametrize("size,eps", [(1e22, 1e-6), (1e-22, 0.0), (1e-19, 0.0), (1e-25, 1e-6)])
def test_kv4_keys_whose_squares_leave_fp32(size, eps):
    """Keys are those of the 64-bit norm, bytes and all, where fp32 could not hold the sum of their squares."""
    from paper_2609_20888_b200 import binding as eb
    rows, d, block = 32, 128, 32
    q, k, v = inputs(rows, 2, 2, d, "fp32", 9)
    k = k * size
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 1000
    w = torch.rand(d, device="cuda") + 0.5
    inv = (10000.0 ** -(torch.arange(64, dtype=torch.float64) / 64)).cuda()
    pool = torch.zeros((1, 2, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
    desc, kv4 = eb.kv4_cache_desc(pool, 2, d, block, batch=1, t_cap=block)
    q_out = torch.empty((rows, 2, d), dtype=torch.bfloat16, device="cuda")
    eb.eta_append_tokens_kv4(desc, kv4, q, k, v, torch.arange(rows, device="cuda"), pos, q_out, pool, inv_freq=inv, k_weight=w, eps=eps)
    _, _, yk, _, _ = expected(q, k, v, pos, None, w, inv, False, eps)
    c, s = ref.encode(yk, 1.0)
    kc, ks, _, _ = ref.split(pool.cpu().numpy(), block, d)
    assert np.array_equal(kc[0], c.transpose(1, 0, 2)) and np.array_equal(ks[0], s.transpose(1, 0, 2))


@pytest.mark.parametrize("four", [False, True])
def test_far_positions_keep_their_angle(four):
    """Positions up to the last 32-bit one, frequencies from 1 down: bytes, or bf16 values, of the 64-bit angle."""
    from paper_2609_20888_b200 import binding as eb
    rows, d, block = 64, 128, 64
    q, k, v = inputs(rows, 1, 1, d, "fp32", 3)
    pos = torch.tensor([0, 1, 105614, 105616, (1 << 24) + 1, (1 << 31) - 1, -1, -100000] + [7919 * 10007 + 123457 * i for i in range(56)],
                       dtype=torch.int32, device="cuda")
    inv = (500000.0 ** -(torch.arange(64, dtype=torch.float64) / 64)).cuda()
    slots = torch.arange(rows, device="cuda")
    q_out = torch.empty((rows, 1, d), dtype=torch.bfloat16, device="cuda")
    yq, sq, yk, sk, _ = expected(q, k, v, pos, None, None, inv, False)
    if four:
        pool = torch.zeros((1, 1, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
        desc, kv4 = eb.kv4_cache_desc(pool, 1, d, block, batch=1, t_cap=block)
        eb.eta_append_tokens_kv4(desc, kv4, q, k, v, slots, pos, q_out, pool, inv_freq=inv)
        kc, ks, _, _ = ref.split(pool.cpu().numpy(), block, d)
        c, s = ref.encode(yk[:, 0], 1.0)
        assert np.array_equal(kc[0, 0], c) and np.array_equal(ks[0, 0], s)
    else:
        K, V = (torch.zeros((1, 1, block, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        eb.eta_append_tokens(eb.cache_desc(K, V, 1, block), q, k, v, slots, pos, q_out, K, V, inv_freq=inv)
        close(K[0, 0], yk[:, 0], sk[:, 0])
    close(q_out, yq, sq)


@pytest.mark.parametrize("four", [False, True])
def test_a_slot_past_the_cache_is_skipped_and_reported(four):
    from paper_2609_20888_b200 import binding as eb
    d, block, pages = 64, 32, 3
    q, k, v = inputs(4, 2, 2, d, "bf16", 1)
    slots = torch.tensor([0, pages * block, 1 << 40, pages * block - 1], device="cuda")
    q_out = torch.full((4, 2, d), 5.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    if four:
        pool = torch.zeros((pages, 2, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
        desc, kv4 = eb.kv4_cache_desc(pool, 2, d, block, batch=1, t_cap=block)
        eb.eta_append_tokens_kv4(desc, kv4, q, k, v, slots, None, q_out, pool, status=status)
    else:
        K, V = (torch.zeros((pages, 2, block, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        eb.eta_append_tokens(eb.paged_cache_desc(K, V, 1, 2, t_cap=block), q, k, v, slots, None, q_out, K, V, paged=True, status=status)
        assert torch.equal(K[0, :, 0], k[0]) and torch.equal(V[2, :, 31], v[3]) and int((K != 0).any(-1).sum()) == 4
    assert status.item() == 8
    assert (q_out[1:3] == 5).all() and torch.equal(q_out[[0, 3]], q[[0, 3]])


def test_captured_on_another_stream_gives_the_same_bytes():
    from paper_2609_20888_b200 import binding as eb
    case = CASES[2]
    q, k, v, pos, wq, wk, inv, slots, n, pages, t_cap, interleaved, hq, hkv, d, block, paged = _setup(case, 13)
    pools = [torch.zeros((pages, hkv, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.zeros((len(slots), hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    desc, kv4 = eb.kv4_cache_desc(pools[0], hq, d, block, batch=3, t_cap=block)
    call = lambda m: eb.eta_append_tokens_kv4(desc, kv4, q, k, v, slots, pos, outs[m], pools[m], inv_freq=inv, q_weight=wq, k_weight=wk)  # noqa: E731
    call(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(1)
        graph.replay()
    side.synchronize()
    assert torch.equal(pools[0], pools[1]) and torch.equal(outs[0], outs[1]) and pools[0].any()


def test_refusals_of_the_binding():
    from paper_2609_20888_b200 import binding as eb
    d, block = 64, 32
    q, k, v = inputs(4, 2, 2, d, "bf16", 1)
    slots, pos, inv = torch.arange(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    q_out = torch.zeros((4, 2, d), dtype=torch.bfloat16, device="cuda")
    K, V = (torch.zeros((1, 2, block, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    desc = eb.cache_desc(K, V, 2, block)
    ok = dict(q=q, k=k, v=v, slot_map=slots, positions=pos, q_out=q_out, K=K, V=V, inv_freq=inv)
    eb.eta_append_tokens(desc, **ok)
    eb.eta_append_tokens(desc, **{**ok, "q": q[:0], "k": k[:0], "v": v[:0], "slot_map": slots[:0], "positions": pos[:0], "q_out": q_out[:0]})
    wide = torch.zeros((2, 2, 2 * block, d), dtype=torch.bfloat16, device="cuda")
    for bad, what in [(dict(q=q.double()), "q"), (dict(k=k.half()), "k"), (dict(v=v[:3]), "v"), (dict(slot_map=slots.int()), "slot_map"),
                      (dict(slot_map=slots[:3]), "slot_map"), (dict(q_out=q_out.float()), "q_out"), (dict(q_out=q_out.transpose(0, 1)), "q_out"),
                      (dict(K=wide), "K"), (dict(V=wide[:1, :, ::2]), "V"), (dict(inv_freq=inv.float()), "inv_freq"),
                      (dict(inv_freq=torch.ones(40, dtype=torch.float64, device="cuda")), "inv_freq"), (dict(positions=pos[:2]), "positions"),
                      (dict(positions=None), "invalid"), (dict(inv_freq=inv[:5]), "unsupported"), (dict(q_weight=torch.ones(32, device="cuda")), "q_weight"),
                      (dict(status=torch.zeros(2, dtype=torch.int32, device="cuda")), "status"), (dict(q=q[..., ::2]), "q")]:
        with pytest.raises(eb.EtaError, match=what):
            eb.eta_append_tokens(desc, **{**ok, **bad})
    pool = torch.zeros((2, 2, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
    d4, kv4 = eb.kv4_cache_desc(pool, 2, d, block, batch=1, t_cap=block)
    how = (d4, kv4, q, k, v, slots, pos, q_out)
    eb.eta_append_tokens_kv4(*how, pool)
    for bad in (pool[:, :1], pool[..., :-16], pool.float(), None, torch.cat((pool, pool), -1)[..., :pool.shape[-1]]):
        with pytest.raises((eb.EtaError, TypeError)):
            eb.eta_append_tokens_kv4(*how, bad)
    with pytest.raises((eb.EtaError, TypeError)):
        eb.eta_append_tokens_kv4(d4, None, *how[2:], pool)
    with pytest.raises(eb.EtaError):
        eb.eta_unpack_kv4(d4, kv4, pool, K, V)                    # one page for two
