"""Prompts and the pages they leave behind: more operators of a serving step, as measurable cases.

Four kinds:

  prompt   attention of a step's new tokens (whole prompts, chunks of them, single tokens; packed, each sequence behind its own
           context) over a bf16 cache that holds them already: softmax, or the gated attention of a sparse decode step with
           every token attended
  fork     sequences that begin as copies of others: full pages are shared, the last partly filled one is copied, and so are the
           block summaries
  free     finished sequences let go of their pages, which go back when nobody else holds them
  compact  pages move to the low end of the pool, in the tables and in memory

`run` computes a case with elementary torch operations, or, where `own` is set, through the framework's entry points.

A sequence's lengths are part of a case (`_lengths`, `_tree`), not drawn: `work` counts them exactly.
"""
from __future__ import annotations

import math

import torch

own = False

# ------------------------------------------------------------------------------------------------------------ cases

_PROMPT = {"kind": "prompt", "batch": 1, "n_q_heads": 32, "n_kv_heads": 8, "head_dim": 128, "block": 64, "new": 8192, "spread": False,
           "context": 0, "single_share": 0.0, "paged": False, "mode": "dense", "beta": 5.0, "ungate": False, "pad": 0, "refused": False}
_FORK = {"kind": "fork", "batch": 16, "parents": 1, "n_kv_heads": 8, "head_dim": 128, "block": 64, "context": 4096, "take": False,
         "layers": 1, "packed": False, "slack": 1.2}
_FREE = {"kind": "free", "batch": 64, "parents": 16, "block": 64, "context": 4096, "release_share": 0.25, "take": False, "slack": 1.3}
_COMPACT = {"kind": "compact", "batch": 64, "parents": 16, "n_kv_heads": 8, "head_dim": 128, "block": 64, "context": 4096,
            "release_share": 0.3, "take": False, "slack": 1.3, "layers": 1}


def listed():
    return [
        # the smallest prompt, of the smallest configuration: latency only
        {"name": "prompt_257", **_PROMPT, "n_q_heads": 8, "n_kv_heads": 2, "head_dim": 64, "block": 32, "new": 257},
        # one prompt of 8K, softmax
        {"name": "prompt_8k", **_PROMPT},
        # packed prompts of odd lengths into a paged cache, gated as the model was trained, rows padded, one sequence turned away
        {"name": "prompt_packed_gated", **_PROMPT, "batch": 11, "new": 4999, "spread": True, "paged": True, "mode": "tau", "ungate": True,
         "pad": 37, "refused": True},
        # two chunks of a long prompt behind what is cached already, pages of 32 tokens, head_dim 64
        {"name": "prompt_chunks_32k", **_PROMPT, "batch": 2, "n_q_heads": 16, "n_kv_heads": 4, "head_dim": 64, "block": 32, "new": 1111,
         "context": 32768, "paged": True, "mode": "const"},
        # continuous batching: single tokens of running requests beside chunks of new ones
        {"name": "prompt_mixed_b64", **_PROMPT, "batch": 64, "new": 600, "spread": True, "context": 16384, "single_share": 0.9, "paged": True},
        # the largest: one prompt of 32K
        {"name": "prompt_32k", **_PROMPT, "new": 32768},
        # eight samples of one prompt of odd length
        {"name": "fork_samples_8", **_FORK, "batch": 9, "context": 2077},
        # a large batch of requests that share the head of a few long prompts, two layers, packed summaries
        {"name": "fork_prefix_b240", **_FORK, "batch": 240, "parents": 12, "context": 32768, "take": True, "layers": 2, "packed": True},
        # a step's finished requests
        {"name": "free_b64", **_FREE},
        # many long forked sequences at once
        {"name": "free_b800", **_FREE, "batch": 800, "parents": 80, "context": 32768, "release_share": 0.5},
        # a small pool of short sequences
        {"name": "compact_b16", **_COMPACT, "batch": 16, "parents": 4, "n_kv_heads": 2, "head_dim": 64, "block": 32, "context": 1024},
        # a pool of gigabytes after a third of its sequences have gone
        {"name": "compact_b64", **_COMPACT, "context": 16384},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "prompt", "fork", "fork", "free", "compact"])
    G, hkv = rng.choice([1, 2, 4, 4, 8]), rng.choice([2, 4, 8])
    d, b = rng.choice([64, 128, 128]), rng.choice([32, 64, 64, 128])
    if kind == "prompt":
        most = {k: v for c in listed() if c["name"] == "prompt_32k" for k, v in work(c).items()}
        case = {**_PROMPT, "batch": _log_int(rng, 1, 64), "n_q_heads": G * hkv, "n_kv_heads": hkv, "head_dim": d, "block": b,
                "new": _log_int(rng, 1, 16384), "spread": rng.random() < 0.6, "context": rng.choice([0, 0, _log_int(rng, 30, 65536)]),
                "single_share": rng.choice([0.0, 0.0, 0.5, 0.95]), "paged": rng.random() < 0.6,
                "mode": rng.choice(["dense", "dense", "tau", "const"]), "beta": rng.choice([5.0, 5.0, 2.0]), "ungate": rng.random() < 0.4,
                "pad": rng.choice([0, rng.randint(1, 100)]), "refused": rng.random() < 0.3}
        while case["batch"] > 1 and (work(case)["flops"] > most["flops"] / 4 or work(case)["bytes"] > 4e9):
            case["batch"] //= 2
        while work(case)["flops"] > most["flops"] / 4:
            case["new"] = case["new"] * 2 // 3
        return case
    parents = _log_int(rng, 1, 40)
    batch = parents + _log_int(rng, 1, 500)
    context = _log_int(rng, 20, 32768)
    tree = {"batch": batch, "parents": parents, "block": b, "context": context, "take": rng.random() < 0.5}
    if kind == "free":
        return {**_FREE, **tree, "release_share": round(rng.uniform(0.02, 1.0), 2), "slack": round(rng.uniform(1.0, 2.0), 2)}
    layers = rng.choice([1, 1, 2])
    while tree["parents"] * tree["context"] * hkv * d * layers > 12 * 32768 * 8 * 128:
        tree["context"] = tree["context"] // 2
    while tree["batch"] > tree["parents"] + 1 and tree["batch"] * (tree["context"] // b + 1) * hkv * d * layers > 240 * 512 * 8 * 128 * 2:
        tree["batch"] = tree["parents"] + (tree["batch"] - tree["parents"]) // 2
    if kind == "fork":
        return {**_FORK, **tree, "n_kv_heads": hkv, "head_dim": d, "layers": layers, "packed": rng.random() < 0.4,
                "slack": rng.choice([1.0, 1.2, 1.5])}
    return {**_COMPACT, **tree, "n_kv_heads": hkv, "head_dim": d, "layers": layers, "release_share": round(rng.uniform(0.05, 0.9), 2),
            "slack": round(rng.uniform(1.0, 2.0), 2)}


# ----------------------------------------------------------------------------------------------------------- lengths

def _frac(i, k):
    """A number in [0, 1) that spreads evenly over i; k selects one of several such sequences."""
    return ((i + 1) * (0.6180339887498949, 0.7548776662466927, 0.5698402909980532)[k]) % 1.0


def _lengths(case):
    """New tokens and tokens cached before them, of every sequence of a prompt case; how many of the new ones were granted."""
    new, before = [], []
    for i in range(case["batch"]):
        one = _frac(i, 0) < case["single_share"]
        new.append(1 if one else (1 + int(_frac(i, 1) * case["new"]) if case["spread"] else case["new"]))
        before.append(int(case["context"] * (0.5 + 0.5 * _frac(i, 2))) if case["batch"] > 1 else case["context"])
    turned_away = [case["refused"] and case["batch"] > 1 and i == case["batch"] // 2 for i in range(case["batch"])]
    return new, before, [0 if r else n for n, r in zip(new, turned_away)]


def _tree(case):
    """Length of every sequence (parents first, then their forks) and the parent of each (-1: none).  Forks have a whole parent, or,
    with `take`, a part of it."""
    P = case["parents"]
    lens = [max(1, int(case["context"] * (0.5 + 0.5 * _frac(i, 1)))) for i in range(P)]
    lens[0] = case["context"]
    parent = [-1] * P
    for i in range(P, case["batch"]):
        parent.append((i * 7) % P)
        lens.append(max(1, int(lens[parent[i]] * (0.2 + 0.8 * _frac(i, 0)))) if case["take"] else lens[parent[i]])
    return lens, parent


def _parent_pages(case, lens):
    b = case["block"]
    return sum(-(-n // b) for n in lens[:case["parents"]])


# ------------------------------------------------------------------------------------------------------------ inputs

def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _prepare_prompt(case, gen):
    B, Hq, Hkv, d, b = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "block"))
    new, before, granted = _lengths(case)
    # a sequence that got nothing has its context only
    lens = [c + g for c, g in zip(before, granted)]
    NB = max(1, -(-max(lens) // b))
    rows = sum(new)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    s = {"row_start": _ints(starts), "lens": _ints(lens), "granted": _ints(granted) if case["refused"] else None,
         "status": _ints([0]), "out": torch.zeros((rows + case["pad"], Hq, d), dtype=torch.bfloat16, device="cuda")}
    # keys about a direction of their head, queries that lean to it: scores of a few units, as trained heads have
    lean = randn(Hkv, 1, d)
    s["q"] = (1.4 * randn(rows + case["pad"], Hkv, Hq // Hkv, d) + 0.5 * lean).reshape(-1, Hq, d).to(torch.bfloat16)
    held = [-(-n // b) for n in lens]
    if case["paged"]:
        pages = sum(held) + 3
        perm = torch.randperm(pages, generator=gen, device="cuda").int()
        s["table"] = torch.full((B, NB), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(held):
            s["table"][i, :n] = perm[at:at + n]
            at += n
        shape = (pages, Hkv, b, d)
    else:
        shape = (B, Hkv, NB * b, d)
    s["K"], s["V"] = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for i in range(0, shape[0], 64):
        n = min(64, shape[0] - i)
        s["K"][i:i + n] = randn(n, *shape[1:]) + 0.3 * lean
        s["V"][i:i + n] = randn(n, *shape[1:])
    s["tau"] = 0.4 * randn(rows + case["pad"], Hq) + 0.5 if case["mode"] == "tau" else None
    s["const"] = 0.4 * randn(Hq) + 0.5 if case["mode"] == "const" else None
    if own:
        from paper_2609_20888_b200 import binding as eb
        if case["paged"]:
            s["desc"] = eb.paged_cache_desc(s["K"], s["V"], B, Hq, t_cap=NB * b)
            s["pages"] = eb.page_table(s["table"], shape[0])
        else:
            s["desc"], s["pages"] = eb.cache_desc(s["K"], s["V"], Hq, b), None
        flags = (eb.ETA_FLAG_DENSE if case["mode"] == "dense" else 0) | (eb.ETA_FLAG_UNGATE_LAST if case["ungate"] else 0)
        s["params"] = eb.DecodeParams(beta=case["beta"], flags=flags)
        n = eb.eta_prefill_workspace_bytes(s["desc"])
        ws = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
        s["ws"] = ws[-ws.data_ptr() % 256:][:n]
    return s


def _prepare_tree(case, gen, forked):
    """Tables, shared counts and the free stack of a pool whose parents, and with `forked` also their forks, hold pages."""
    b, P = case["block"], case["parents"]
    lens, parent = _tree(case)
    NB = -(-max(lens) // b)
    tails = sum(1 for n in lens[P:] if n % b)
    used = _parent_pages(case, lens) + (tails if forked else 0)
    pages = max(used + 1, int((_parent_pages(case, lens) + tails) * case["slack"]))
    perm = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((case["batch"], NB), -1, dtype=torch.int32, device="cuda")
    shared = torch.zeros(pages, dtype=torch.int32, device="cuda")
    at = 0
    for i in range(case["batch"] if forked else P):
        n = -(-lens[i] // b)
        whole = 0
        if parent[i] >= 0:
            whole = lens[i] // b
            table[i, :whole] = table[parent[i], :whole]
        table[i, whole:n] = perm[at:at + n - whole]
        at += n - whole
    held = torch.arange(NB, device="cuda") < -(-_ints(lens) // b)[:, None]
    if not forked:
        held[P:] = False
    shared += (torch.bincount(table[held].long(), minlength=pages) - 1).clamp(min=0).int()
    free = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    free[:pages - at] = perm[at:]
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"lens": _ints([n if forked or i < P else 0 for i, n in enumerate(lens)]), "table": table, "shared": shared, "free": free,
            "n_free": _ints([pages - at]), "t_cap": NB * b, "lens_out": ints(case["batch"]), "shared_out": ints(pages), "n_free_out": ints(1),
            "status": ints(1)}


def _pools(case, pages, gen):
    shape = (pages, case["n_kv_heads"], case["block"], case["head_dim"])
    pools = []
    for _ in range(2 * case["layers"]):
        pools.append(torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen))
    return pools


def _prepare_fork(case, gen):
    s = _prepare_tree(case, gen, False)
    lens, parent = _tree(case)
    B, d = case["batch"], case["head_dim"]
    NB = s["table"].shape[1]
    s["parent"], s["take"] = _ints(parent), _ints(lens) if case["take"] else None
    s["pools"] = _pools(case, s["shared"].numel(), gen)
    rows = (B, case["n_kv_heads"], NB)
    s["musig"], s["mnorm"] = [], []
    for _ in range(case["layers"]):
        if case["packed"]:
            s["musig"].append(torch.randint(0, 120, (*rows, 3 * d), generator=gen, device="cuda", dtype=torch.uint8))
        else:
            s["musig"].append(torch.randn((*rows, 2, d), generator=gen, device="cuda").half())
        s["mnorm"].append(torch.rand(rows, generator=gen, device="cuda"))
    for k in ("copy_src", "copy_dst", "got"):
        s[k] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if own:
        from paper_2609_20888_b200 import binding as eb
        s["desc"] = eb.paged_cache_desc(s["pools"][0], s["pools"][1], B, case["n_kv_heads"], t_cap=s["t_cap"])
    return s


def _workspace(s):
    from paper_2609_20888_b200 import binding as eb
    n = eb.eta_pages_workspace_bytes(s["shared"].numel())
    ws = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
    return ws[-ws.data_ptr() % 256:][:n]


def _prepare_free(case, gen):
    s = _prepare_tree(case, gen, True)
    s["release"] = (torch.rand(case["batch"], generator=gen, device="cuda") < case["release_share"]).int()
    if own:
        s["ws"] = _workspace(s)
    return s


def _prepare_compact(case, gen):
    s = _prepare_tree(case, gen, True)
    # some sequences have gone already
    s["release"] = (torch.rand(case["batch"], generator=gen, device="cuda") < case["release_share"]).int()
    _free(s)
    s["lens"], s["shared"], s["n_free"] = s["lens_out"].clone(), s["shared_out"].clone(), s["n_free_out"].clone()
    s["pools"] = _pools(case, s["shared"].numel(), gen)
    pages = s["shared"].numel()
    s["table_out"], s["free_out"] = torch.zeros_like(s["table"]), torch.full_like(s["free"], -1)
    s["move_src"], s["move_dst"] = (torch.full((pages,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    s["n_moves"] = _ints([0])
    if own:
        s["ws"] = _workspace(s)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"prompt": _prepare_prompt, "fork": _prepare_fork, "free": _prepare_free, "compact": _prepare_compact}
    s = make[case["kind"]](case, gen)
    s["case"] = case
    return s


# ------------------------------------------------------------------------------------------------------- plain forms

def _prompt(s):
    case, b = s["case"], s["case"]["block"]
    Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    new, before, granted = _lengths(case)
    row0 = 0
    for i, n in enumerate(new):
        if not granted[i]:
            row0 += n
            continue
        T = before[i] + n
        if case["paged"]:
            pages = s["table"][i, :-(-T // b)].long()
            K, V = (x[pages].transpose(0, 1).flatten(1, 2).float() for x in (s["K"], s["V"]))
        else:
            K, V = s["K"][i].float(), s["V"][i].float()
        step = max(1, 2 ** 28 // (Hq * T))
        for r in range(0, n, step):
            m = min(step, n - r)
            end = before[i] + r + m
            at = slice(row0 + r, row0 + r + m)
            q = s["q"][at].float().reshape(m, Hkv, -1, d).permute(1, 2, 0, 3)
            score = (q @ K[:, None, :end].transpose(2, 3)).div_(math.sqrt(d))                # [Hkv, G, m, end]
            p = torch.arange(end - m, end, device="cuda")[:, None]
            t = torch.arange(end, device="cuda")
            if case["mode"] != "dense":
                cut = s["tau"][at].t().reshape(Hkv, -1, m, 1) if case["mode"] == "tau" else s["const"].reshape(Hkv, -1, 1, 1)
                gate = torch.sigmoid((score - cut).mul_(case["beta"]))
                if case["ungate"]:
                    gate.masked_fill_(t == p, 1.0)
                score.mul_(gate)
            score.masked_fill_(t > p, -math.inf)
            score.sub_(score.amax(3, keepdim=True)).exp_()
            out = (score @ V[:, None, :end]) / score.sum(3, keepdim=True)
            s["out"][at] = out.permute(2, 0, 1, 3).reshape(m, Hq, d).to(torch.bfloat16)
        row0 += n


def _fork(s):
    case, b = s["case"], s["case"]["block"]
    lens, parent = s["lens"], s["parent"].long()
    j = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    child = parent >= 0
    of = parent.clamp(min=0)
    T = torch.where(child, lens[of], 0)
    if s["take"] is not None:
        T = torch.minimum(T, s["take"])
    whole, tail = T // b, (T % b != 0) & child
    nth = torch.cumsum(tail, 0).int() - tail.int()
    ok = child & (~tail | (nth < s["n_free"]))
    mine = tail & ok
    page = s["free"][(s["n_free"] - 1 - nth).clamp(min=0).long()]
    shares = (j < whole[:, None]) & ok[:, None]
    theirs = s["table"][of]
    s["copy_src"].copy_(torch.where(mine, theirs.gather(1, whole.clamp(max=j.numel() - 1)[:, None].long())[:, 0], -1))
    s["copy_dst"].copy_(torch.where(mine, page, -1))
    table = torch.where(shares, theirs, s["table"])
    s["table"].copy_(torch.where((j == whole[:, None]) & mine[:, None], page[:, None], table))
    s["shared_out"].copy_(s["shared"] + torch.bincount(theirs[shares].long(), minlength=s["shared"].numel()).int())
    s["got"].copy_(torch.where(ok, T, 0))
    s["lens_out"].copy_(torch.where(ok, T, lens))
    s["n_free_out"].copy_(s["n_free"] - mine.sum(dtype=torch.int32))
    src, dst = s["copy_src"][mine].long(), s["copy_dst"][mine].long()
    for pool in s["pools"]:
        pool[dst] = pool[src]
    take = (j < (s["got"] // b)[:, None]) & child[:, None]
    i, k = torch.nonzero(take, as_tuple=True)
    for musig, mnorm in zip(s["musig"], s["mnorm"]):
        musig[i, :, k] = musig[of[i], :, k]
        mnorm[i, :, k] = mnorm[of[i], :, k]


def _free(s):
    b = s["t_cap"] // s["table"].shape[1]
    j = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    gone = (j < -(-s["lens"] // b)[:, None]) & (s["release"] != 0)[:, None]
    count = torch.bincount(s["table"][gone].long(), minlength=s["shared"].numel()).int()
    back = torch.nonzero(count > s["shared"])[:, 0]
    s["free"][s["n_free"].long() + torch.arange(back.numel(), device="cuda")] = back.int()
    s["shared_out"].copy_((s["shared"] - count).clamp(min=0))
    s["lens_out"].copy_(torch.where(s["release"] != 0, 0, s["lens"]))
    s["n_free_out"].copy_(s["n_free"] + back.numel())


def _compact(s):
    case, b = s["case"], s["case"]["block"]
    pages = s["shared"].numel()
    number = torch.arange(pages, device="cuda", dtype=torch.int32)
    free = torch.zeros(pages, dtype=torch.bool, device="cuda")
    free[s["free"][number < s["n_free"]].long()] = True
    live = pages - s["n_free"]
    dst = torch.nonzero(free & (number < live))[:, 0].int()
    src = torch.nonzero(~free & (number >= live))[:, 0].int()
    n = src.numel()
    s["move_src"][:n] = src
    s["move_dst"][:n] = dst
    s["n_moves"].fill_(n)
    to = number.clone()
    to[src.long()] = dst
    j = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    held = j < -(-s["lens"] // b)[:, None]
    s["table_out"].copy_(torch.where(held, to[s["table"].clamp(min=0).long()], s["table"]))
    shared = s["shared"].clone()
    shared[src.long()] = 0
    shared[dst.long()] = s["shared"][src.long()]
    s["shared_out"].copy_(shared)
    s["free_out"].copy_(torch.where(number < s["n_free"], pages - 1 - number, s["free_out"]))
    s["n_free_out"].copy_(s["n_free"])
    for pool in s["pools"]:
        pool[dst.long()] = pool[src.long()]


# -------------------------------------------------------------------------------------------------------------- pass

def _own_pass(s):
    from paper_2609_20888_b200 import binding as eb
    case, kind = s["case"], s["case"]["kind"]
    if kind == "prompt":
        eb.eta_prefill(s["desc"], s["params"], s["q"], s["K"], s["V"], s["row_start"], s["lens"], s["out"], s["ws"], tau=s["tau"],
                       head_const=s["const"], granted=s["granted"], status=s["status"], pages=s["pages"])
    elif kind == "fork":
        eb.eta_fork_pages(case["block"], s["t_cap"], s["parent"], s["lens"], s["table"], s["shared"], s["free"], s["n_free"], s["copy_src"],
                          s["copy_dst"], s["got"], take=s["take"], seq_lens_out=s["lens_out"], shared_out=s["shared_out"],
                          n_free_out=s["n_free_out"], status=s["status"])
        eb.eta_copy_pages(s["pools"], s["copy_src"], s["copy_dst"], status=s["status"])
        for musig, mnorm in zip(s["musig"], s["mnorm"]):
            eb.eta_fork_summaries(s["desc"], s["parent"], s["got"], musig, mnorm, status=s["status"])
    elif kind == "free":
        eb.eta_free_pages(s["t_cap"] // s["table"].shape[1], s["t_cap"], s["release"], s["lens"], s["table"], s["shared"], s["free"],
                          s["n_free"], s["ws"], seq_lens_out=s["lens_out"], shared_out=s["shared_out"], n_free_out=s["n_free_out"],
                          status=s["status"])
    else:
        eb.eta_compact_pages(case["block"], s["t_cap"], s["lens"], s["table"], s["shared"], s["free"], s["n_free"], s["move_src"],
                             s["move_dst"], s["n_moves"], s["ws"], block_table_out=s["table_out"], shared_out=s["shared_out"],
                             free_pages_out=s["free_out"], n_free_out=s["n_free_out"], status=s["status"])
        eb.eta_copy_pages(s["pools"], s["move_src"], s["move_dst"], n_moves=s["n_moves"], status=s["status"])


_OUTPUTS = {"prompt": ("out",),
            "fork": ("table", "shared_out", "lens_out", "n_free_out", "got", "copy_src", "copy_dst", "pools", "musig", "mnorm"),
            "free": ("free", "shared_out", "lens_out", "n_free_out"),
            "compact": ("table_out", "shared_out", "free_out", "n_free_out", "move_src", "move_dst", "n_moves", "pools")}


def run(state):
    kind = state["case"]["kind"]
    if own:
        _own_pass(state)
    else:
        {"prompt": _prompt, "fork": _fork, "free": _free, "compact": _compact}[kind](state)
    return {k: state[k] for k in _OUTPUTS[kind]}


# ------------------------------------------------------------------------------------------------------------- floor

def work(case):
    """Bytes and operations that a pass cannot do without."""
    b = case["block"]
    if case["kind"] == "prompt":
        new, before, granted = _lengths(case)
        Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
        pairs = sum(g * c + g * (g + 1) // 2 for g, c in zip(granted, before))
        rows, tokens = sum(granted), sum(c + g for g, c in zip(granted, before) if g)
        return {"bytes": 4 * rows * Hq * d + 4 * tokens * Hkv * d + (4 * rows * Hq if case["mode"] == "tau" else 0),
                "flops": 4 * d * Hq * pairs}
    lens, parent = _tree(case)
    P, held = case["parents"], [-(-n // b) for n in lens]
    if case["kind"] == "fork":
        tails = sum(1 for n in lens[P:] if n % b)
        whole = sum(n // b for n in lens[P:])
        page = 4 * case["n_kv_heads"] * b * case["head_dim"] * case["layers"]
        record = ((3 if case["packed"] else 4) * case["head_dim"] + 4) * case["n_kv_heads"] * case["layers"]
        distinct = sum(max(lens[i] // b for i in range(P, case["batch"]) if parent[i] == p) if p in parent else 0 for p in range(P))
        return {"bytes": 2 * page * tails + record * (whole + distinct) + 4 * (whole + distinct) + 20 * case["batch"], "flops": 0}
    tails = sum(1 for n in lens[P:] if n % b)
    if case["kind"] == "free":
        gone = case["release_share"] * sum(held)
        return {"bytes": 4 * gone + 8 * (_parent_pages(case, lens) + tails) + 12 * case["batch"], "flops": 0}
    # how many pages move: those that sit above the line once the released are gone, at the mean
    r = case["release_share"]
    used = [-(-lens[p] // b) for p in range(P)]
    kids = [sum(1 for i in range(P, case["batch"]) if parent[i] == p) for p in range(P)]
    live = sum(n * (1 - r ** (1 + k)) for n, k in zip(used, kids)) + tails * (1 - r)
    total = max(sum(used) + tails + 1, int((sum(used) + tails) * case["slack"]))
    page = 4 * case["n_kv_heads"] * b * case["head_dim"] * case["layers"]
    return {"bytes": 2 * page * live * (1 - live / total) + 8 * sum(held) + 16 * total, "flops": 0}


# ------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    if case["kind"] != "prompt":
        return None
    s = prepare(case, seed)
    Hq, Hkv, d, b = (case[k] for k in ("n_q_heads", "n_kv_heads", "head_dim", "block"))
    G = Hq // Hkv
    out = s["out"].double()
    starts, lens = s["row_start"].tolist(), s["lens"].tolist()
    for i in range(case["batch"]):
        n, T = starts[i + 1] - starts[i], lens[i]
        if s["granted"] is not None and int(s["granted"][i]) == 0:
            continue
        for h in range(Hkv):
            if case["paged"]:
                at = torch.arange(T, device="cuda")
                pages = s["table"][i].long()[at // b]
                K, V = s["K"][pages, h, at % b].double(), s["V"][pages, h, at % b].double()
            else:
                K, V = s["K"][i, h, :T].double(), s["V"][i, h, :T].double()
            step = max(1, 2 ** 27 // (T * G))
            for r in range(0, n, step):
                rows = torch.arange(r, min(n, r + step), device="cuda")
                p = T - n + rows
                end = int(p[-1]) + 1
                q = s["q"][starts[i] + rows, h * G:(h + 1) * G].double().transpose(0, 1)                  # [G, rows, d]
                S = torch.matmul(q, K[:end].T) * d ** -0.5
                see = torch.arange(end, device="cuda")[None] <= p[:, None]
                if case["mode"] != "dense":
                    cut = (s["tau"][starts[i] + rows, h * G:(h + 1) * G].double().T if case["mode"] == "tau"
                           else s["const"][h * G:(h + 1) * G].double()[:, None].expand(G, rows.numel()))
                    gated = S / (1 + torch.exp(-case["beta"] * (S - cut[:, :, None])))
                    if case["ungate"]:
                        own_token = torch.arange(end, device="cuda")[None] == p[:, None]
                        gated = torch.where(own_token, S, gated)
                    S = gated
                S = torch.where(see, S, -math.inf)
                w = torch.exp(S - torch.logsumexp(S, 2, keepdim=True))
                out[starts[i] + rows, h * G:(h + 1) * G] = torch.matmul(w, V[:end]).transpose(0, 1)
    return {"out": out}
