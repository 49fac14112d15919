"""Operators around the KV cache of a serving step, as measurable cases.

Four kinds, in the order in which a step makes them:

  plan    block tables and slot maps from request lengths: pages of finished sequences go back, new tokens get pages
  tokens  the step's queries, keys and values: norm per head, rotation by position, queries stored, keys and values written
          to the cache (bf16, or 4 bits; of the latter what the cache then stands for is read back in the same pass)
  index   block summaries of a 4-bit cache: all of them (prefill), or of the blocks that the newest tokens completed
  attend  one decode step's screening and attention over a 4-bit cache

`run` computes a case with elementary torch operations, or, where `own` is set, through the framework's entry points.

The 4-bit cache: a block of `block` tokens of one KV head is one run of bytes, K codes [block][d / 2], K scales [block][d / 16], V
codes, V scales.  A code is a 4-bit float (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; channel 2 j in the low half of byte j), a scale
an 8-bit float (e4m3) shared by 16 channels; a value is code * scale * the tensor's own scale g.  A group x is stored with the scale
e4m3(max|x| / (6 g)) and the codes e2m1(x / (scale g)): quotients rounded to fp32, then to the nearest, ties to even.
"""
from __future__ import annotations

import math

import torch

own = False

# ------------------------------------------------------------------------------------------------------------ cases

_PLAN = {"kind": "plan", "batch": 64, "block": 64, "context": 16384, "new": 1, "prefill_share": 0.0, "release_share": 0.0, "pad": 0}
_TOKENS = {"kind": "tokens", "rows": 8, "n_q_heads": 32, "n_kv_heads": 8, "head_dim": 128, "block": 64, "dtype": "bf16", "bits": 16,
           "paged": True, "norm": True, "rotary": 128, "interleaved": False, "run": 1, "far": 131072, "pad": 0, "g": 1.0}
_INDEX = {"kind": "index", "batch": 4, "n_kv_heads": 8, "head_dim": 128, "block": 64, "context": 131072, "min_context": 0, "paged": False,
          "newest": False, "g": 1.0}
_ATTEND = {"kind": "attend", "batch": 1, "n_q_heads": 32, "n_kv_heads": 8, "head_dim": 128, "block": 64, "context": 2048,
           "min_context": 0, "sparsity": 0.9, "dense": False, "frozen": False, "paged": False, "lwb": 0, "beta": 5.0, "g": 1.0}


def listed():
    return [
        # every decode step of a server: one token for each of 64 running requests
        {"name": "plan_decode_b64", **_PLAN},
        # continuous batching at its heaviest: long prompts beside decoding requests, finished ones replaced, a padded row count
        {"name": "plan_prefill_b200", **_PLAN, "batch": 200, "new": 9000, "prefill_share": 0.4, "release_share": 0.25, "pad": 4099},
        # the new tokens of a small decode batch
        {"name": "tokens_decode_b8", **_TOKENS},
        # a prefill chunk of odd length into a paged bf16 cache
        {"name": "tokens_prefill_8k", **_TOKENS, "rows": 8229, "run": 2743},
        # a large decode batch into a 4-bit cache: head_dim 64, half of it rotated in neighbouring pairs, fp16, padded rows
        {"name": "tokens_kv4_decode_b128", **_TOKENS, "rows": 128, "n_q_heads": 32, "n_kv_heads": 4, "head_dim": 64, "dtype": "fp16",
         "bits": 4, "rotary": 32, "interleaved": True, "pad": 16, "g": 0.75},
        # four prompts of 8K into a 4-bit cache with a row per sequence
        {"name": "tokens_kv4_prefill_32k", **_TOKENS, "rows": 32768, "bits": 4, "paged": False, "run": 8192, "far": 8192},
        # the blocks that a decode step of 64 sequences completes
        {"name": "kv4_append_b64", **_INDEX, "batch": 64, "context": 4096, "newest": True, "paged": True},
        # prefill of the headline batch
        {"name": "kv4_build_b4_128k", **_INDEX},
        # the smallest configuration: latency only
        {"name": "kv4_attend_2k", **_ATTEND, "n_q_heads": 8, "n_kv_heads": 2, "head_dim": 64, "block": 32, "sparsity": 0.7},
        # a small serving batch of odd length, paged
        {"name": "kv4_attend_b8_32k", **_ATTEND, "batch": 8, "context": 32768 + 77, "sparsity": 0.84, "paged": True, "lwb": 4, "g": 0.75},
        # the headline cache with 90 % of its blocks screened out
        {"name": "kv4_attend_b4_128k_s90", **_ATTEND, "batch": 4, "context": 131072},
        # every block attended, ungated: 16 sequences of mixed lengths, eight query heads to a KV head
        {"name": "kv4_attend_dense_b16", **_ATTEND, "batch": 16, "n_kv_heads": 4, "context": 65536, "min_context": 8192, "dense": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "tokens", "tokens", "index", "attend", "attend", "attend"])
    G, hkv = rng.choice([1, 2, 4, 4, 8]), rng.choice([2, 4, 8])
    d, b = rng.choice([64, 128, 128]), rng.choice([32, 64, 64, 128])
    g = rng.choice([1.0, 1.0, 0.75, 1.5, 0.40625])
    if kind == "plan":
        share = rng.choice([0.0, round(rng.uniform(0.05, 0.4), 2)])
        batch = _log_int(rng, 1, 1500)
        new = _log_int(rng, 2, max(3, min(16384, int(700000 / max(1, batch * max(share, 0.05)))))) if share else 1
        return {**_PLAN, "batch": batch, "block": b, "context": _log_int(rng, 200, 32768), "new": new, "prefill_share": share,
                "release_share": rng.choice([0.0, round(rng.uniform(0.02, 0.3), 2)]), "pad": rng.choice([0, rng.randint(1, 300)])}
    if kind == "tokens":
        rows = _log_int(rng, 1, 32768 * 4 // hkv)
        rows = max(1, min(rows, 32768 * 40 * 128 // ((G + 2) * hkv * d)))
        run = rng.choice([1, _log_int(rng, 1, rows)])
        run = max(run, -(-rows // 256))
        return {**_TOKENS, "rows": rows, "n_q_heads": G * hkv, "n_kv_heads": hkv, "head_dim": d, "block": b,
                "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "bits": rng.choice([16, 4]), "paged": rng.random() < 0.6,
                "norm": rng.random() < 0.7, "rotary": rng.choice([d, d, d // 2, 0]), "interleaved": rng.random() < 0.4, "run": run,
                "far": _log_int(rng, run, max(run + 1, 65536)), "pad": rng.choice([0, rng.randint(1, 40) % rows]), "g": g}
    context = _log_int(rng, 40 if kind == "attend" else 2 * b, 256 * 1024)
    batch = _log_int(rng, 1, 64)
    while batch > 1 and batch * hkv * context * d > 4 * 8 * 131072 * 128:
        batch //= 2
    mixed = batch > 1 and rng.random() < 0.5
    lens = {"batch": batch, "n_kv_heads": hkv, "head_dim": d, "block": b, "context": context,
            "min_context": max(1, context // 8) if mixed else 0, "paged": rng.random() < 0.5, "g": g}
    if kind == "index":
        return {**_INDEX, **lens, "newest": rng.random() < 0.3}
    return {**_ATTEND, **lens, "n_q_heads": G * hkv, "sparsity": round(rng.uniform(0.5, 0.97), 2), "dense": rng.random() < 0.25,
            "frozen": rng.random() < 0.3, "lwb": rng.choice([0, 0, 1, 4]), "beta": rng.choice([5.0, 5.0, 2.0])}


# --------------------------------------------------------------------------------------------------- the 4-bit cache

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _block_bytes(block, d):
    return 2 * block * (d // 2 + d // 16)


def _views(blocks, block, d):
    """K codes, K scales, V codes, V scales of blocks uint8 [..., block bytes]: views [..., block, d / 2] and [..., block, d / 16]."""
    c, s = block * (d // 2), block * (d // 16)
    at = (0, c, c + s, 2 * c + s, 2 * c + 2 * s)
    return tuple(blocks[..., at[k]:at[k + 1]].unflatten(-1, (block, -1)) for k in range(4))


def _decoded(codes, scales, g, dtype=torch.float32):
    """[..., d] values."""
    table = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), dtype=dtype, device=codes.device)
    value = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    s = scales.view(torch.float8_e4m3fn).to(dtype)
    return (value.unflatten(-1, (-1, 16)) * (s * g)[..., None]).flatten(-2)


def _coded(x, g):
    """codes, scales of x [..., d] (64 bits: a value next to a border goes the way its formula says)."""
    x = x.double().unflatten(-1, (-1, 16))
    scales = (x.abs().amax(-1) / (6 * g)).float().clamp(max=448).to(torch.float8_e4m3fn)
    unit = (scales.double() * g)[..., None]
    y = torch.where(unit > 0, x / unit.clamp(min=1e-300), torch.zeros_like(x)).float()
    m = y.abs()
    code = (m > 0.25).byte() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
    code = (code | torch.signbit(y).byte() << 3).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales.view(torch.uint8)


# ------------------------------------------------------------------------------------------------------------ inputs

_DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _lens(case, gen):
    lens = torch.full((case["batch"],), case["context"], dtype=torch.int32, device="cuda")
    if case["min_context"]:
        lens = torch.randint(case["min_context"], case["context"] + 1, lens.shape, generator=gen, device="cuda", dtype=torch.int32)
        lens[0] = case["context"]
    return lens


def _plan_rows(case):
    """Rows of the buffers, which a program sizes once: a tenth more than the mean step has."""
    return int(case["batch"] * (1 + 1.1 * case["prefill_share"] * case["new"])) + case["pad"]


def _prepare_plan(case, gen):
    B, b = case["batch"], case["block"]
    rand = lambda n: torch.rand(n, generator=gen, device="cuda")  # noqa: E731
    lens = (1 + rand(B) * case["context"]).int()
    new = torch.ones(B, dtype=torch.int32, device="cuda")
    prefill = rand(B) < case["prefill_share"]
    new = torch.where(prefill, (1 + rand(B) * case["new"] * 2).int(), new)
    new = torch.where(rand(B) < 0.05, 0, new) if case["prefill_share"] else new
    release = (rand(B) < case["release_share"]).int()
    stride = -(-(case["context"] + 2 + 2 * case["new"]) // b)
    held = -(-lens // b)
    perm = torch.randperm(B * stride, generator=gen, device="cuda").int()
    before = torch.cumsum(held, 0) - held
    j = torch.arange(stride, device="cuda", dtype=torch.int32)
    table = torch.where(j < held[:, None], perm[(before[:, None] + j).clamp(max=B * stride - 1)], -1)
    free = torch.full((B * stride,), -1, dtype=torch.int32, device="cuda")
    used = int(held.sum())
    free[:B * stride - used] = perm[used:]
    rows = _plan_rows(case)
    ints = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
    return {"lens": lens, "new": new, "release": release if case["release_share"] else None, "table": table, "free": free,
            "n_free": torch.tensor([B * stride - used], dtype=torch.int32, device="cuda"), "rows": rows, "t_cap": stride * b,
            "slots": ints(rows, torch.int64), "positions": ints(rows), "row_start": ints(B + 1), "granted": ints(B),
            "lens_out": ints(B), "n_free_out": ints(1), "status": ints(1)}


def _prepare_tokens(case, gen):
    R, Hq, Hkv, d, b, run = (case[k] for k in ("rows", "n_q_heads", "n_kv_heads", "head_dim", "block", "run"))
    dtype = _DTYPE[case["dtype"]]
    # one projection holds a row's queries, keys and values
    qkv = torch.randn((R, Hq + 2 * Hkv, d), generator=gen, device="cuda")
    qkv[:, Hq:Hq + Hkv] *= 1 + 3 * torch.rand((Hkv, d), generator=gen, device="cuda")       # keys have channels that stand out
    qkv = qkv.to(dtype)
    # sequences of `run` new tokens each, a start of its own for each
    n_seq = -(-R // run)
    start = torch.randint(0, max(1, case["far"] - run + 1), (n_seq,), generator=gen, device="cuda")
    seq = torch.arange(R, device="cuda") // run
    positions = start[seq] + torch.arange(R, device="cuda") % run
    s = {"q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + Hkv], "v": qkv[:, Hq + Hkv:], "positions": positions.int(),
         "q_out": torch.zeros((R, Hq, d), dtype=torch.bfloat16, device="cuda"),
         "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    # where the rows go: only the blocks that the call writes to are here
    first = start // b
    need = (run + b - 2) // b + 1
    local = positions - (first * b)[seq]
    if case["paged"]:
        pages = n_seq * need
        perm = torch.randperm(pages, generator=gen, device="cuda")
        page = perm[seq * need + local // b]
        s["slots"] = page * b + local % b
        shape = (pages, Hkv)
    else:
        s["slots"] = seq * (need * b) + local
        shape = (n_seq, Hkv, need)
    if case["pad"]:
        s["slots"][R - case["pad"]:] = -1
    kv = (shape[0], Hkv, (1 if case["paged"] else shape[2]) * b, d)
    s["K"], s["V"] = (torch.zeros(kv, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if case["bits"] == 4:
        s["pool"] = torch.zeros((*shape, _block_bytes(b, d)), dtype=torch.uint8, device="cuda")
    s["wq"], s["wk"] = ((1 + 0.2 * torch.randn((2, d), generator=gen, device="cuda")).unbind(0)) if case["norm"] else (None, None)
    half = case["rotary"] // 2
    s["inv_freq"] = 500000.0 ** -(torch.arange(half, device="cuda", dtype=torch.float64) / half) if half else None
    if own:
        from paper_2609_20888_b200 import binding as eb
        if case["bits"] == 4:
            s["desc"], s["kv4"] = eb.kv4_cache_desc(s["pool"], Hq, d, b, batch=n_seq, t_cap=kv[2], k_scale=case["g"], v_scale=case["g"])
        elif case["paged"]:
            s["desc"] = eb.paged_cache_desc(s["K"], s["V"], n_seq, Hq, t_cap=b)
        else:
            s["desc"] = eb.cache_desc(s["K"], s["V"], Hq, b)
    return s


def _prepare_cache(case, gen):
    """A 4-bit cache of clustered keys, its lengths and, where it is paged, its table."""
    B, Hkv, d, b = case["batch"], case["n_kv_heads"], case["head_dim"], case["block"]
    NB = -(-case["context"] // b)
    s = {"lens": _lens(case, gen)}
    if case.get("newest"):
        s["lens"] = ((s["lens"] + b - 1) // b * b).int()          # the newest token completes a block, but for one sequence in eight
        s["lens"][::8] -= 1
    blocks = torch.empty((B, Hkv, NB, _block_bytes(b, d)), dtype=torch.uint8, device="cuda")
    centroid = torch.randn((Hkv, 64, d), generator=gen, device="cuda")
    for i in range(B):
        which = torch.randint(0, 64, (Hkv, NB), generator=gen, device="cuda")
        mean = torch.gather(centroid, 1, which[:, :, None].expand(-1, -1, d))[:, :, None]
        # an fp32 pass is enough here: the bytes are the input
        for at, x in ((0, mean + 0.3 * torch.randn((Hkv, NB, b, d), generator=gen, device="cuda")),
                      (2, torch.randn((Hkv, NB, b, d), generator=gen, device="cuda"))):
            views = _views(blocks[i], b, d)
            for h in range(Hkv):
                views[at][h], views[at + 1][h] = _coded(x[h] * case["g"], case["g"])
    s["pool"] = blocks
    if case["paged"]:
        perm = torch.randperm(B * NB, generator=gen, device="cuda")
        s["pool"] = torch.empty((B * NB, Hkv, blocks.shape[-1]), dtype=torch.uint8, device="cuda")
        s["pool"][perm] = blocks.transpose(1, 2).flatten(0, 1)
        s["table"] = perm.view(B, NB).int()
    if own:
        from paper_2609_20888_b200 import binding as eb
        s["desc"], s["kv4"] = eb.kv4_cache_desc(s["pool"], case.get("n_q_heads", Hkv), d, b, batch=B, t_cap=NB * b, k_scale=case["g"],
                                                v_scale=case["g"])
        s["pages"] = eb.page_table(s["table"], B * NB) if case["paged"] else None
    return s


def _prepare_index(case, gen):
    s = _prepare_cache(case, gen)
    B, Hkv, d = case["batch"], case["n_kv_heads"], case["head_dim"]
    NB = -(-case["context"] // case["block"])
    s["musig"] = torch.zeros((B, Hkv, NB, 2, d), dtype=torch.float16, device="cuda")
    s["mnorm"] = torch.zeros((B, Hkv, NB), device="cuda")
    return s


def _bounds(q, musig, mnorm, z=1.0):
    """Score_dual: [B, Hkv, G, NB] of queries [B, Hkv, G, d]."""
    mu, sigma = musig.to(q.dtype).unbind(3)
    moment = q @ mu.transpose(2, 3) + z * (q.square() @ sigma.square().transpose(2, 3)).sqrt()
    sphere = q.square().sum(3, keepdim=True).sqrt() * mnorm.to(q.dtype)[:, :, None]
    return torch.minimum(moment, sphere) / math.sqrt(q.shape[3])


def _thresholds(case, bounds, full):
    """Per head and sequence (frozen: per head), in the middle of the widest gap near the place where the union over a KV head's query
    heads keeps 1 - sparsity of the blocks: which survive does not hang on a bound's last bit."""
    B, Hkv, G, NB = bounds.shape
    rel = bounds.masked_fill(~full[:, None, None], -math.inf).reshape(B, Hkv * G, NB)
    if case["frozen"]:
        rel = rel.transpose(0, 1).reshape(1, Hkv * G, B * NB)
    ranked = rel.sort(2, descending=True).values
    n = torch.isfinite(ranked).sum(2, keepdim=True)
    if int(n.max()) < 2:
        return torch.zeros(ranked.shape[:2], device="cuda")
    last = (n - 2).clamp(min=0)
    lo, hi = 0.0, 1.0
    for _ in range(12):
        mid = (lo + hi) / 2
        cut = ranked.gather(2, torch.minimum((mid * n).long(), last))
        kept = ((rel >= cut) & torch.isfinite(rel)).view(*rel.shape[:1], Hkv, G, -1).any(2).sum() / (n.view(-1, Hkv, G)[:, :, 0].sum())
        lo, hi = (mid, hi) if float(kept) < 1 - case["sparsity"] else (lo, mid)
    w = max(2, int(n.max()) // 100)
    near = torch.minimum(((hi * n).long() + torch.arange(-w, w + 1, device="cuda")).clamp(min=0), last)
    gap = ranked.gather(2, near) - ranked.gather(2, near + 1)
    best = near.gather(2, gap.nan_to_num(-1, -1, -1).argmax(2, keepdim=True))
    tau = ((ranked.gather(2, best) + ranked.gather(2, best + 1)) / 2)[..., 0]
    return torch.where(torch.isfinite(tau), tau, 0).contiguous()


def _prepare_attend(case, gen):
    s = _prepare_cache(case, gen)
    B, Hq, Hkv, d, b = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "block"))
    NB = -(-case["context"] // b)
    # the heads of a KV group share a direction, as grouped heads do
    shared = torch.randn((B, Hkv, 1, d), generator=gen, device="cuda")
    noise = torch.randn((B, Hkv, Hq // Hkv, d), generator=gen, device="cuda")
    s["q"] = ((math.sqrt(0.95) * shared + math.sqrt(0.05) * noise) / case["g"]).reshape(B, Hq, d).to(torch.bfloat16)
    s["musig"] = torch.zeros((B, Hkv, NB, 2, d), dtype=torch.float16, device="cuda")
    s["mnorm"] = torch.zeros((B, Hkv, NB), device="cuda")
    for i in range(B):
        codes, scales = (x[0] for x in _cache_views(s, case, slice(i, i + 1))[:2])
        for h in range(Hkv):
            _summaries(_decoded(codes[h], scales[h], case["g"]), s["musig"][i, h], s["mnorm"][i, h])
    full = torch.arange(NB, device="cuda") < (s["lens"] // b)[:, None]
    s["musig"] *= full[:, None, :, None, None]
    s["mnorm"] *= full[:, None]
    cut = _thresholds(case, _bounds(s["q"].double().view(B, Hkv, -1, d), s["musig"], s["mnorm"]), full).float()
    s["tau"], s["const"] = (None, cut[0].contiguous()) if case["frozen"] else (cut, None)
    s["out"] = torch.zeros((B, Hq, d), device="cuda")
    s["sel"] = torch.zeros((B, Hkv, NB), dtype=torch.uint8, device="cuda")
    s["stats"] = torch.zeros((B, Hkv), dtype=torch.int32, device="cuda")
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2609_20888_b200 import binding as eb
        s["params"] = eb.DecodeParams(beta=case["beta"], lwb=case["lwb"], flags=eb.ETA_FLAG_DENSE if case["dense"] else 0)
        n = eb.eta_kv4_workspace_bytes(s["desc"])
        ws = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
        s["ws"] = ws[-ws.data_ptr() % 256:][:n]
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"plan": _prepare_plan, "tokens": _prepare_tokens, "index": _prepare_index, "attend": _prepare_attend}
    return {"case": case, **make[case["kind"]](case, gen)}


# ------------------------------------------------------------------------------------------------------- plain forms

def _plan(s):
    case, b, stride = s["case"], s["case"]["block"], s["table"].shape[1]
    j = torch.arange(stride, device="cuda", dtype=torch.int32)
    lens, n_free = s["lens"], s["n_free"]
    if s["release"] is not None:
        # finished sequences hand their pages back, in order
        gone = torch.where(s["release"] != 0, -(-lens // b), 0)
        to = n_free + (torch.cumsum(gone, 0) - gone)[:, None] + j
        back = j < gone[:, None]
        s["free"][to[back].long()] = s["table"][back]
        lens = torch.where(s["release"] != 0, 0, lens)
        n_free = n_free + gone.sum(dtype=torch.int32)
    new = s["new"].clamp(min=0)
    row_start = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0)).int()
    fits = (lens + new <= s["t_cap"]) & (row_start[1:] <= s["rows"])
    held, want = -(-lens // b), -(-(lens + new) // b)
    need = torch.where(fits, want - held, 0)
    upto = torch.cumsum(need, 0)
    ok = fits & ((need == 0) | (upto <= n_free))
    take = torch.where(ok, need, 0)
    s["granted"].copy_(torch.where(ok, new, 0))
    s["lens_out"].copy_(lens + s["granted"])
    s["row_start"].copy_(row_start)
    # pages come off the end of the free list, sequence after sequence
    at = n_free - 1 - (torch.cumsum(take, 0) - take)[:, None] - (j - held[:, None])
    fresh = (j >= held[:, None]) & (j < (held + take)[:, None])
    s["table"].copy_(torch.where(fresh, s["free"][at.clamp(min=0).long()], s["table"]))
    s["n_free_out"].copy_(n_free - take.sum(dtype=torch.int32))
    row = torch.arange(s["rows"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["row_start"][1:], row, right=True).clamp(max=case["batch"] - 1)
    pos = lens[seq] + row - row_start[seq]
    live = (row < row_start[-1]) & (s["granted"][seq] > 0)
    pos = torch.where(live, pos, 0)
    page = s["table"][seq, (pos // b).long()].long()
    s["slots"].copy_(torch.where(live, page * b + pos % b, -1))
    s["positions"].copy_(pos)


def _normed(x, w, eps, dtype):
    x = x.to(dtype)
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w.to(dtype)


def _rotated(x, s):
    n = s["case"]["rotary"]
    if not n:
        return x
    angle = s["positions"].double()[:, None, None] * s["inv_freq"]
    cos, sin = angle.cos().to(x.dtype), angle.sin().to(x.dtype)
    if s["case"]["interleaved"]:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :n // 2], x[..., n // 2:n]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, x[..., n:]), -1)


def _tokens(s):
    case, b = s["case"], s["case"]["block"]
    here = torch.nonzero(s["slots"] >= 0)[:, 0]
    q = _rotated(_normed(s["q"], s["wq"], 1e-6, torch.float32), s)
    s["q_out"][here] = q[here].to(torch.bfloat16)
    # what is about to be held in four bits is decided in 64
    k = _rotated(_normed(s["k"], s["wk"], 1e-6, torch.float64 if case["bits"] == 4 else torch.float32), s)[here]
    v, slots = s["v"][here], s["slots"][here]
    if case["bits"] == 16:
        per = s["K"].shape[2]
        s["K"][slots // per, :, slots % per] = k.to(torch.bfloat16)
        s["V"][slots // per, :, slots % per] = v.to(torch.bfloat16)
        return
    blocks = s["pool"] if case["paged"] else s["pool"].transpose(1, 2)
    views = _views(blocks, b, case["head_dim"])
    if case["paged"]:
        at = (slots // b, slice(None), slots % b)
    else:
        per = s["pool"].shape[2] * b
        at = (slots // per, slots % per // b, slice(None), slots % b)
    for x, codes, scales in ((k, *views[:2]), (v, *views[2:])):
        codes[at], scales[at] = _coded(x, case["g"])
    views = _views(s["pool"], b, case["head_dim"])
    for to, codes, scales in ((s["K"], *views[:2]), (s["V"], *views[2:])):
        to.copy_(_decoded(codes, scales, case["g"]).reshape(to.shape))


def _cache_views(s, case, seqs=slice(None)):
    """K codes, K scales, V codes, V scales of sequences: [B, Hkv, NB, block, ..]"""
    blocks = s["pool"][s["table"][seqs].long()].transpose(1, 2) if case["paged"] else s["pool"][seqs]
    return _views(blocks, case["block"], case["head_dim"])


def _summaries(k, musig, mnorm):
    """Mean and population deviation of every block of k [..., NB, block, d], and the largest norm."""
    var, mean = torch.var_mean(k, -2, correction=0)
    musig.copy_(torch.stack((mean, var.sqrt()), -2))
    mnorm.copy_(k.square().sum(-1).amax(-1).sqrt())


def _index(s):
    case, b = s["case"], s["case"]["block"]
    j = torch.arange(s["mnorm"].shape[2], device="cuda")
    codes, scales = _cache_views(s, case)[:2]
    nb = (s["lens"] // b)[:, None]
    if case["newest"]:
        done = (s["lens"] > 0) & (s["lens"] % b == 0)
        at = (nb[:, 0] - 1).clamp(min=0).long()
        i = torch.arange(case["batch"], device="cuda")
        codes, scales = codes[i, :, at][:, :, None], scales[i, :, at][:, :, None]
        write = done[:, None] & (j == at[:, None])
    else:
        write = j < nb
    k = _decoded(codes, scales, case["g"])
    musig = torch.empty((*k.shape[:3], 2, k.shape[-1]), dtype=torch.float16, device="cuda")
    mnorm = torch.empty(k.shape[:3], device="cuda")
    _summaries(k, musig, mnorm)
    s["musig"].copy_(torch.where(write[:, None, :, None, None], musig, s["musig"]))
    s["mnorm"].copy_(torch.where(write[:, None], mnorm, s["mnorm"]))


def _admitted(case, bounds, cut, full, window=128):
    """Which blocks each head attends: those whose bound is not below the threshold, the newest lwb, and the best of the first
    `window` where a head has none of those."""
    if case["dense"]:
        return full.expand_as(bounds)
    j = torch.arange(bounds.shape[3], device="cuda")
    n = full.sum(-1, keepdim=True)
    keep = full & (~(bounds < cut[..., None]) | (j >= n - case["lwb"]))
    first = full & (j < window)
    best = bounds.masked_fill(~first, -math.inf).argmax(3, keepdim=True)
    none = ~(keep & first).any(3, keepdim=True) & (n > 0)
    return keep | (none & (j == best))


def _attend(s):
    case, b = s["case"], s["case"]["block"]
    B, Hkv, d = case["batch"], case["n_kv_heads"], case["head_dim"]
    q = s["q"].float().view(B, Hkv, -1, d)
    T = s["lens"][:, None, None, None]
    j = torch.arange(s["sel"].shape[2], device="cuda")
    cut = (s["const"].view(1, Hkv, -1) if case["frozen"] else s["tau"].view(B, Hkv, -1)).expand(B, Hkv, q.shape[2])
    keep = _admitted(case, _bounds(q, s["musig"], s["mnorm"]), cut, j < T // b)
    bit = 2 ** torch.arange(q.shape[2], device="cuda")
    s["sel"].copy_((keep * bit[:, None]).sum(2))
    s["stats"].copy_(keep.any(2).sum(2))
    kc, ks, vc, vs = _cache_views(s, case)
    score = q @ _decoded(kc, ks, case["g"]).flatten(2, 3).transpose(2, 3) / math.sqrt(d)
    if not case["dense"]:
        score = score * torch.sigmoid(case["beta"] * (score - cut[..., None]))
    t = torch.arange(score.shape[3], device="cuda")
    live = (keep.repeat_interleave(b, 3) | (t >= T // b * b)) & (t < T)
    p = torch.softmax(score.masked_fill(~live, -math.inf), 3)
    s["out"].copy_((p @ _decoded(vc, vs, case["g"]).flatten(2, 3)).reshape(s["out"].shape))


# -------------------------------------------------------------------------------------------------------------- pass

def _own_pass(s):
    from paper_2609_20888_b200 import binding as eb
    case, kind = s["case"], s["case"]["kind"]
    if kind == "plan":
        eb.eta_plan_pages(case["block"], s["t_cap"], s["new"], s["lens"], s["table"], s["free"], s["n_free"], s["slots"], s["positions"],
                          s["row_start"], s["granted"], seq_lens_out=s["lens_out"], n_free_out=s["n_free_out"], release=s["release"],
                          status=s["status"])
    elif kind == "tokens":
        how = {"inv_freq": s["inv_freq"], "q_weight": s["wq"], "k_weight": s["wk"], "interleaved": case["interleaved"], "status": s["status"]}
        if case["bits"] == 16:
            eb.eta_append_tokens(s["desc"], s["q"], s["k"], s["v"], s["slots"], s["positions"], s["q_out"], s["K"], s["V"],
                                 paged=case["paged"], **how)
        else:
            eb.eta_append_tokens_kv4(s["desc"], s["kv4"], s["q"], s["k"], s["v"], s["slots"], s["positions"], s["q_out"], s["pool"], **how)
            eb.eta_unpack_kv4(s["desc"], s["kv4"], s["pool"], s["K"], s["V"])
    elif kind == "index":
        call = eb.eta_append_summary_kv4 if case["newest"] else eb.eta_build_block_summaries_kv4
        call(s["desc"], s["kv4"], s["pool"], s["lens"], s["musig"], s["mnorm"], pages=s["pages"])
    else:
        eb.eta_decode_kv4(s["desc"], s["kv4"], s["params"], s["q"], s["pool"], s["lens"], s["musig"], s["mnorm"], s["tau"], s["const"],
                          s["out"], s["sel"], s["ws"], stats=s["stats"], status=s["status"], pages=s["pages"])


_OUTPUTS = {"plan": ("slots", "positions", "row_start", "granted", "lens_out", "n_free_out", "table", "free"),
            "tokens": ("q_out", "K", "V"), "index": ("musig", "mnorm"), "attend": ("out", "sel", "stats")}


def run(state):
    kind = state["case"]["kind"]
    if own:
        _own_pass(state)
    else:
        {"plan": _plan, "tokens": _tokens, "index": _index, "attend": _attend}[kind](state)
    return {k: state[k] for k in _OUTPUTS[kind]}


# ------------------------------------------------------------------------------------------------------------- floor

def work(case):
    """Bytes and operations that a pass cannot do without, at the mean length of a mixed batch."""
    b = case["block"]
    if case["kind"] == "plan":
        rows = _plan_rows(case)
        pages = rows / b
        gone = case["batch"] * case["release_share"] * case["context"] / 2 / b
        return {"bytes": 12 * rows + 8 * pages + 8 * gone + 24 * case["batch"], "flops": 0}
    Hkv, d = case["n_kv_heads"], case["head_dim"]
    record = d // 2 + d // 16
    if case["kind"] == "tokens":
        Hq = case["n_q_heads"]
        rows = case["rows"] - case["pad"]
        read = (4 if case["dtype"] == "fp32" else 2) * (Hq + 2 * Hkv) * d + 12
        held = -(-case["rows"] // case["run"]) * ((case["run"] + b - 2) // b + 1) * b
        written = 4 * Hkv * d if case["bits"] == 16 else 2 * Hkv * record
        readback = 0 if case["bits"] == 16 else held * Hkv * (2 * record + 4 * d)
        return {"bytes": rows * (read + 2 * Hq * d + written) + readback, "flops": rows * (Hq + Hkv) * d * 8}
    B = case["batch"]
    T = (case["min_context"] + case["context"]) / 2 if case["min_context"] else case["context"]
    blocks = B * Hkv * (1 if case["kind"] == "index" and case["newest"] else T // b)
    if case["kind"] == "index":
        return {"bytes": blocks * (b * record + 4 * d + 4), "flops": blocks * b * d * 6}
    G = case["n_q_heads"] // Hkv
    screen = 0 if case["dense"] else blocks * (4 * d + 4)
    tokens = blocks * (1 if case["dense"] else 1 - case["sparsity"]) * b + B * Hkv * (T % b)
    return {"bytes": screen + blocks + 2 * record * tokens + 6 * B * Hkv * G * d,
            "flops": (0 if case["dense"] else 4 * d * blocks * G) + 4 * d * G * tokens}


# ------------------------------------------------------------------------------------------------------- in 64 bits

def _exact_codes(x, g):
    """The values that a 4-bit cache holds for x [..., d], from the definition: nearest of the sixteen to x / (scale g)."""
    x = x.double().reshape(*x.shape[:-1], -1, 16)
    e4m3 = torch.arange(127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()
    want = (x.abs().amax(-1) / (6 * g)).float().double()
    up = torch.searchsorted(e4m3, want).clamp(max=126)
    down = (up - 1).clamp(min=0)
    gap = (want - e4m3[down]) - (e4m3[up] - want)
    scale = e4m3[torch.where((gap > 0) | ((gap == 0) & (up % 2 == 0)), up, down)] * g
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    y = torch.where(scale[..., None] > 0, x / scale[..., None], 0).float().double()
    up = torch.searchsorted(grid, y.abs().contiguous()).clamp(max=7)
    down = (up - 1).clamp(min=0)
    gap = (y.abs() - grid[down]) - (grid[up] - y.abs())
    code = torch.where((gap > 0) | ((gap == 0) & (up % 2 == 0)), up, down)
    return (torch.copysign(grid[code], x) * scale[..., None]).flatten(-2)


def _exact_values(codes, scales, g):
    """Code bytes and scale bytes to values, from the fields of the two formats."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    e, m = c // 2 % 4, (c % 2).double()
    value = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1)) * (1 - 2 * (c // 8))
    s = scales.long()
    scale = torch.where(s // 8 == 0, (s % 8).double() / 512, (1 + (s % 8).double() / 8) * 2.0 ** (s // 8 - 7))
    return value * scale.repeat_interleave(16, -1) * g


def _exact_tokens(case, s):
    n, live = case["rotary"], s["slots"] >= 0
    result = {"q_out": s["q_out"].double(), "K": s["K"].double(), "V": s["V"].double()}
    slots = s["slots"][live]

    def made(x, w):
        x = x.double()[live]
        if w is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * w.double()
        if n:
            angle = torch.outer(s["positions"][live].double(), s["inv_freq"])[:, None]
            pair = x[..., :n].unflatten(-1, (n // 2, 2) if case["interleaved"] else (2, n // 2))
            z = torch.view_as_complex((pair if case["interleaved"] else pair.transpose(-1, -2)).contiguous())
            z = torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle))
            x = torch.cat(((z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2), x[..., n:]), -1)
        return x

    result["q_out"][live] = made(s["q"], s["wq"])
    for name, x in (("K", made(s["k"], s["wk"])), ("V", s["v"].double()[live])):
        per = result[name].shape[2]
        result[name][slots // per, :, slots % per] = x if case["bits"] == 16 else _exact_codes(x, case["g"])
    return result


def _exact_blocks(s, case, i):
    """K, V of sequence i in 64 bits: [Hkv, NB * block, d]."""
    b, d = case["block"], case["head_dim"]
    raw = (s["pool"][s["table"][i].long()].transpose(0, 1) if case["paged"] else s["pool"][i]).contiguous()
    c, e = b * d // 2, b * d // 16
    kc, ks, vc, vs = raw.split((c, e, c, e), -1)
    return tuple(_exact_values(x.reshape(*x.shape[:2], b, -1), y.reshape(*y.shape[:2], b, -1), case["g"]).flatten(1, 2)
                 for x, y in ((kc, ks), (vc, vs)))


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    if case["kind"] == "tokens":
        return _exact_tokens(case, s)
    b, d, Hkv = case["block"], case["head_dim"], case["n_kv_heads"]
    if case["kind"] == "index":
        musig, mnorm = s["musig"].double(), s["mnorm"].double()
        for i in range(case["batch"]):
            n = int(s["lens"][i]) // b
            at = range(n)
            if case["newest"]:
                at = [n - 1] if n and int(s["lens"][i]) % b == 0 else []
            if not len(at):
                continue
            at = torch.tensor(list(at), device="cuda")
            k = _exact_blocks(s, case, i)[0].unflatten(1, (-1, b))[:, at]
            mean = k.sum(2) / b
            musig[i, :, at, 0] = mean
            musig[i, :, at, 1] = ((k - mean[:, :, None]) ** 2).sum(2).div(b).sqrt()
            mnorm[i, :, at] = k.norm(dim=3).amax(2)
        return {"musig": musig, "mnorm": mnorm}
    out = s["out"].double()
    for i in range(case["batch"]):
        T = int(s["lens"][i])
        n = T // b
        K, V = _exact_blocks(s, case, i)
        for h in range(Hkv):
            G = case["n_q_heads"] // Hkv
            q = s["q"][i, h * G:(h + 1) * G].double()
            cut = (s["const"] if case["frozen"] else s["tau"][i])[h * G:(h + 1) * G].double()
            S = K[h, :T] @ q.T / math.sqrt(d)
            live = torch.ones((T, G), dtype=torch.bool, device="cuda")
            if not case["dense"]:
                mu, sigma = s["musig"][i, h, :n].double().unbind(1)
                bound = torch.minimum(mu @ q.T + (sigma.pow(2) @ q.pow(2).T).sqrt(),
                                      s["mnorm"][i, h, :n].double()[:, None] * q.norm(dim=1)) / math.sqrt(d)
                keep = bound >= cut
                keep[max(0, n - case["lwb"]):] = True
                if n:
                    lost = ~keep[:128].any(0)
                    keep[bound[:128].argmax(0)[lost], torch.nonzero(lost)[:, 0]] = True
                live[:n * b] = keep.repeat_interleave(b, 0)
                S = S / (1 + torch.exp(-case["beta"] * (S - cut)))
            S[~live] = -math.inf
            p = torch.exp(S - S.amax(0))
            out[i, h * G:(h + 1) * G] = (p.T @ V[h, :T]) / p.sum(0)[:, None]
    return {"out": out, "sel": None, "stats": None}
