"""Attention of a step's new tokens on a GPU, against 64 bits: head layouts, block sizes, contiguous and paged, lengths from one token to
several tiles, softmax and gate, split and whole items, masked infinities, rows that do not count."""
import math

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from prefill_reference import reference

pytestmark = pytest.mark.gpu
CANARY = 3.25


def make(new, before, Hkv, G, d, b, paged, seed=0, pad=0, granted=None, layout="bhtd", short=()):
    """Sequences of new[i] tokens behind before[i]; `short`: sequences whose length says 5 fewer than they have new tokens."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = len(new)
    lens = [c + (n if granted is None else granted[i]) for i, (n, c) in enumerate(zip(new, before))]
    for i in short:
        lens[i] = max(0, new[i] - 5)
    NB = max(1, -(-max(lens) // b))
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q = randn(starts[-1] + pad, Hkv * G, d).bfloat16() * 1.5
    s = {"q": q, "starts": starts, "lens": lens, "granted": granted, "Hq": Hkv * G}
    if paged:
        held = [-(-n // b) for n in lens]
        pages = sum(held) + 2
        perm = torch.randperm(pages, generator=gen, device="cuda").int()
        table = torch.full((B, NB), 2 ** 30, dtype=torch.int32, device="cuda")     # entries that nobody may follow
        at = 0
        for i, n in enumerate(held):
            table[i, :n] = perm[at:at + n]
            at += n
        shape = (pages, Hkv, b, d)
        s["table"] = table
    else:
        shape = (B, Hkv, NB * b, d)
    if layout == "bhtd":
        K, V = randn(*shape).bfloat16(), randn(*shape).bfloat16()
    else:                                                   # token-major, heads inside
        K, V = (randn(shape[0], shape[2], shape[1], d).bfloat16().transpose(1, 2) for _ in range(2))
    # what no row sees: behind the sequences
    for x in (K, V):
        for i in range(B):
            for t in range(lens[i], min(NB * b, lens[i] + 3 * b)):
                if paged:
                    if t // b >= -(-lens[i] // b):
                        break
                    x[s["table"][i, t // b].item(), :, t % b] = float("nan")
                else:
                    x[i, :, t] = float("nan")
    s.update(K=K, V=V, paged=paged, b=b, NB=NB, d=d, B=B)
    return s


def gather(s, x):
    got = []
    for i in range(s["B"]):
        if s["paged"]:
            pages = s["table"][i, :-(-s["lens"][i] // s["b"])].long()
            got.append(x[pages].transpose(0, 1).flatten(1, 2)[:, :s["lens"][i]])
        else:
            got.append(x[i, :, :s["lens"][i]])
    return got


def workspace(desc):
    n = eb.eta_prefill_workspace_bytes(desc)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")       # whatever was there before: NaN
    return ws[-ws.data_ptr() % 256:][:n]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def call(s, params, tau=None, const=None, out=None, ws=None):
    if s["paged"]:
        desc = eb.paged_cache_desc(s["K"], s["V"], s["B"], s["Hq"], t_cap=s["NB"] * s["b"])
        pages = eb.page_table(s["table"], s["K"].shape[0])
    else:
        desc, pages = eb.cache_desc(s["K"], s["V"], s["Hq"], s["b"]), None
    out = torch.full_like(s["q"], CANARY) if out is None else out
    status = ints([0])
    eb.eta_prefill(desc, params, s["q"], s["K"], s["V"], ints(s["starts"]), ints(s["lens"]), out, workspace(desc) if ws is None else ws, tau=tau,
                   head_const=const, granted=None if s["granted"] is None else ints(s["granted"]), status=status, pages=pages)
    return out, int(status)


def check(s, params, tau=None, const=None, status=0):
    out, got = call(s, params, tau, const)
    assert got == status
    te = None
    if not params.flags & eb.ETA_FLAG_DENSE:
        te = (tau if tau is not None else const.expand(s["q"].shape[0], -1)) - params.a
    scale = params.scale if params.scale > 0 else 1 / math.sqrt(s["d"])
    want, bound, counts = reference(s["q"], gather(s, s["K"]), gather(s, s["V"]), s["starts"], s["lens"], s["granted"], scale, params.beta, te,
                                    bool(params.flags & eb.ETA_FLAG_UNGATE_LAST))
    assert torch.all(out[~counts] == CANARY)
    err, bound = (out.double() - want).abs()[counts], bound[counts]
    assert torch.all(err <= bound), (err / bound).nan_to_num(0).max().item()       # (rows that see nothing are exactly zero)
    return out


DENSE = eb.DecodeParams(flags=eb.ETA_FLAG_DENSE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("b", [32, 64, 128])
def test_one_prompt(d, G, b):
    check(make([197], [0], 2, G, d, b, paged=b == 64, seed=G), DENSE)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(n, d):
    check(make([n], [0], 1, 4, d, 32, paged=n % 2 == 0, seed=n), DENSE)


@pytest.mark.parametrize("before", [1, 31, 127, 128, 129, 1000, 5000])
@pytest.mark.parametrize("n", [1, 70])
def test_behind_a_context(n, before):
    check(make([n], [before], 2, 4, 128, 64, paged=before % 2 == 1, seed=before), DENSE)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("d,G,b", [(128, 4, 64), (64, 8, 32), (128, 1, 128)])
def test_packed(d, G, b, paged):
    """Sequences of all kinds beside each other: none, one token, whole prompts, chunks, one that was turned away, rows behind the last."""
    new = [3, 0, 1, 260, 1, 77, 129, 1, 40]
    before = [0, 500, 900, 0, 64, 333, 128, 0, 2000]
    granted = [3, 0, 1, 260, 1, 0, 129, 1, 40]
    check(make(new, before, 2, G, d, b, paged, seed=3, pad=21, granted=granted), DENSE)


@pytest.mark.parametrize("mode", ["tau", "const"])
@pytest.mark.parametrize("d,G,b,paged", [(128, 4, 64, True), (64, 2, 32, False), (128, 8, 128, False)])
@pytest.mark.parametrize("ungate", [0, eb.ETA_FLAG_UNGATE_LAST])
def test_gate(mode, d, G, b, paged, ungate):
    s = make([150, 1, 300], [0, 700, 90], 2, G, d, b, paged, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    tau = torch.randn((s["q"].shape[0], s["Hq"]), generator=gen, device="cuda") + 0.3
    params = eb.DecodeParams(beta=3.0, a=0.25, scale=0.11, flags=ungate)
    check(s, params, tau=tau if mode == "tau" else None, const=tau[0].contiguous() if mode == "const" else None)


@pytest.mark.parametrize("te", [-math.inf, math.inf, 0.0, 30.0, -30.0])
@pytest.mark.parametrize("beta", [5.0, 0.0])
def test_gate_at_its_ends(te, beta):
    """An open gate is softmax, a closed one weighs every token alike, beta = 0 halves the scores."""
    s = make([140], [60], 1, 4, 128, 64, False, seed=8)
    const = torch.full((4,), te, device="cuda")
    if beta and math.isinf(te):
        out, _ = call(s, eb.DecodeParams(beta=beta), const=const)
        if te < 0:
            want, bound, _ = reference(s["q"], gather(s, s["K"]), gather(s, s["V"]), s["starts"], s["lens"], None, 1 / math.sqrt(128))
        else:
            want, bound, _ = reference(s["q"], gather(s, s["K"]), gather(s, s["V"]), s["starts"], s["lens"], None, 0.0)
        assert ((out.double() - want).abs() <= bound).all()
    elif beta == 0 and math.isinf(te):
        out, _ = call(s, eb.DecodeParams(beta=0.0), const=const)
        want, bound, _ = reference(s["q"], gather(s, s["K"]), gather(s, s["V"]), s["starts"], s["lens"], None, 0.5 / math.sqrt(128))
        assert ((out.double() - want).abs() <= bound).all()
    else:
        check(s, eb.DecodeParams(beta=beta), const=const)


@pytest.mark.parametrize("size", [30.0, 300.0, 3e4, 1e12])
@pytest.mark.parametrize("te", [0.0, 2000.0])
def test_gate_of_large_scores(size, te):
    """Scores on both sides of 2^11, up to which four gates share a reciprocal and none is smaller than 2^-31 (|S| 2^-31, within the bound)."""
    s = make([140], [60], 1, 4, 128, 64, False, seed=22)
    s["q"] = (s["q"].float() * size).bfloat16()
    check(s, eb.DecodeParams(beta=0.5), const=torch.full((4,), te, device="cuda"))


def test_a_threshold_that_is_nan_is_a_row_that_is_nan():
    s = make([70], [0], 1, 4, 128, 64, False, seed=9)
    tau = torch.zeros((70, 4), device="cuda")
    tau[33, 2] = math.nan
    out, _ = call(s, eb.DecodeParams(), tau=tau)
    bad = torch.isnan(out.float())
    assert bad[33, 2].all() and bad.sum() == 128


@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
@pytest.mark.parametrize("paged", [False, True])
def test_cache_layouts(layout, paged):
    check(make([90, 33], [40, 200], 4, 2, 64, 64, paged, seed=11, layout=layout), DENSE)


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [0, 64, 130, 131, 199])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_masked_does_not_reach_a_row(what, at, d):
    """A value in V at one token: rows before it are as if it were not there, rows from it on have it in that channel."""
    s = make([200], [0], 1, 4, d, 64, False, seed=12)
    clean, _ = call(s, DENSE)
    s["V"][0, 0, at, 7] = what
    s["K"][0, 0, 199] = math.nan if math.isnan(what) else s["K"][0, 0, 199]
    out, _ = call(s, DENSE)
    assert torch.equal(out[:at], clean[:at])
    last = 199 if math.isnan(what) else 200
    assert torch.equal(out[at:last, :, :7], clean[at:last, :, :7]) and torch.equal(out[at:last, :, 8:], clean[at:last, :, 8:])
    got = out[at:last, :, 7].float()
    assert torch.isnan(got).all() if math.isnan(what) else (got == what).all()
    if math.isnan(what):
        assert torch.isnan(out[199].float()).all()


def test_infinities_of_both_signs_in_a_split_item():
    s = make([1], [4000], 1, 8, 128, 64, True, seed=13)
    page = s["table"][0, 4000 // 64].item()
    s["V"][page, 0, 4000 % 64, 3] = math.inf
    s["V"][page, 0, 4000 % 64, 4] = -math.inf
    out, _ = call(s, DENSE)
    assert (out[0, :, 3].float() == math.inf).all() and (out[0, :, 4].float() == -math.inf).all()
    assert torch.isfinite(out[0, :, 5:].float()).all()


@pytest.mark.parametrize("gated,size", [(False, 1.0), (True, 1.0), (True, 1e13)])
def test_infinities_on_both_sides_of_a_sequence_that_sees_nothing(gated, size):
    """A long sequence, one whose row has no tokens at all, a short one, over and over: what was taken out of the long one's last tile is not
    forgotten over the short one's, which may be there before the long one's end (with 15 heads they are 16 items apart).  Scores of 10^13: weights
    underflow, and 0 * inf is NaN where the parts of an item are joined; what was forgotten would be finite."""
    H, G, times = 15, 8, 100
    new, lens = [32, 1, 32] * times, [2040, 0, 40] * times
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    gen = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn((3 * times, H, 2048, 64), generator=gen, device="cuda").bfloat16() for _ in range(2))
    V[::3, :, 2030, 5] = V[2::3, :, 35, 5] = math.inf
    q = (torch.randn((starts[-1], H * G, 64), generator=gen, device="cuda") * size).bfloat16()
    p = torch.cat([torch.arange(t - n, t) for n, t in zip(new, lens)]).cuda()          # the rows' positions
    at = torch.cat([torch.full((n,), 2030 if t > 40 else 35) for n, t in zip(new, lens)]).cuda()
    desc = eb.cache_desc(K, V, H * G, 64)
    ws, out, starts, lens, const = workspace(desc), torch.zeros_like(q), ints(starts), ints(lens), torch.zeros(H * G, device="cuda")
    for _ in range(5):
        out.fill_(CANARY)
        eb.eta_prefill(desc, eb.DecodeParams() if gated else DENSE, q, K, V, starts, lens, out, ws, head_const=const if gated else None)
        got = out[p >= at][:, :, 5].float()
        assert (got == math.inf).all() if size == 1.0 else not torch.isfinite(got).any()
        assert torch.isfinite(out[p < at].float()).all() and torch.all(out[p < 0] == 0)
        assert torch.isfinite(out[:, :, 6:].float()).all()


@pytest.mark.parametrize("bad", [-1, 0])
@pytest.mark.parametrize("d", [64, 128])
def test_a_page_outside_the_pool_reads_as_zeros(d, bad):
    """Next to an infinity that is taken out of the same tile and added again: the page's values are not looked for then either."""
    s = make([60], [200], 2, 4, d, 32, True, seed=21)
    s["V"][s["table"][0, 7].item(), :, 16, 7] = math.inf             # token 240, of the tile of 128 .. 255
    pages = s["K"].shape[0]
    spare = [i for i in range(pages) if i not in s["table"][0, :9].tolist()][0]
    s["K"][spare], s["V"][spare] = 0, 0
    for block in (6, 1):
        s["table"][0, block] = spare
    want, _ = call(s, DENSE)
    for block in (6, 1):
        s["table"][0, block] = bad if bad < 0 else pages + block
    out, status = call(s, DENSE)
    assert status == 0 and torch.equal(out, want)
    assert (out[40:, :, 7].float() == math.inf).all() and torch.isfinite(out[:40].float()).all()


@pytest.mark.parametrize("new,n", [(40, 5), (300, 5), (3, 3)])
def test_more_new_tokens_than_the_sequence_has(new, n):
    """The first rows stand before the sequence's first token: zeros, and a flag."""
    s = make([new, 20], [0, 10], 2, 4, 64, 32, False, seed=14, short=[0])
    out = check(s, DENSE, status=eb.ETA_DEV_EMPTY_ROW)
    assert torch.all(out[:n] == 0)


def test_a_length_past_the_capacity_is_clamped():
    s = make([50], [14], 1, 4, 64, 32, False, seed=15)
    want, _ = call(s, DENSE)
    s["lens"] = [1000]
    out, status = call(s, DENSE)
    assert status == eb.ETA_DEV_LEN_CLAMPED and torch.equal(out, want)


@pytest.mark.parametrize("size", [1e4, 1e18])
def test_scores_far_apart(size):
    """Scores of any size: the largest takes all, ties share."""
    s = make([130], [0], 1, 2, 64, 64, False, seed=16)
    s["q"] = (s["q"].float() * size).bfloat16()
    out, _ = call(s, DENSE)
    q, k, v = s["q"].double(), s["K"][0, 0, :130].double(), s["V"][0, 0, :130].double()
    S = torch.einsum("rhd,td->rht", q, k)
    t = torch.arange(130, device="cuda")
    S.masked_fill_(t[None, None] > t[:, None, None], -math.inf)
    top = S.topk(2, dim=2)
    clear = (top.values[..., 0] - top.values[..., 1]) / 8 > 40          # weights of the others below 2^-57
    want = v[top.indices[..., 0]]
    err = (out.double() - want).abs()[clear]
    assert clear.sum() > 200 and (err <= 2.0 ** -8 * want[clear].abs() * 1.01 + 1e-12).all()


def test_many_sequences_of_one_token():
    """Running requests only: split along the cache and joined."""
    gen = torch.Generator().manual_seed(1)
    before = torch.randint(0, 3000, (40,), generator=gen).tolist()
    check(make([1] * 40, before, 2, 4, 128, 64, True, seed=17), DENSE)


def test_a_thousand_sequences():
    gen = torch.Generator().manual_seed(2)
    new = torch.randint(0, 3, (1024,), generator=gen).tolist()
    before = torch.randint(0, 80, (1024,), generator=gen).tolist()
    check(make(new, before, 1, 4, 64, 32, True, seed=18), DENSE)


def test_whole_items_in_rounds():
    """Enough work that no item is split: rounds of whole items, several head groups."""
    check(make([700] * 24, [0] * 24, 4, 1, 64, 64, False, seed=19), DENSE)


@pytest.mark.parametrize("paged", [False, True])
def test_the_same_bits_every_time_and_under_capture(paged):
    s = make([300, 1, 45], [100, 2000, 0], 2, 4, 128, 64, paged, seed=20)
    want, _ = call(s, DENSE)
    desc = eb.paged_cache_desc(s["K"], s["V"], 3, 8, t_cap=s["NB"] * 64) if paged else eb.cache_desc(s["K"], s["V"], 8, 64)
    pages = eb.page_table(s["table"], s["K"].shape[0]) if paged else None
    out, ws = torch.zeros_like(s["q"]), workspace(desc)
    start, lens = ints(s["starts"]), ints(s["lens"])
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            eb.eta_prefill(desc, DENSE, s["q"], s["K"], s["V"], start, lens, out, ws, pages=pages)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_offsets_past_two_to_the_31():
    """A cache of more than 2^31 elements: the last sequence's keys lie past it."""
    B, Hkv, T, d = 3, 4, 1 << 21, 128
    K, V = (torch.zeros((B, Hkv, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens, new = [130, 0, T], [130, 0, 60]
    gen = torch.Generator(device="cuda").manual_seed(3)
    K[2, :, -500:] = torch.randn((Hkv, 500, d), generator=gen, device="cuda").bfloat16() + 2
    V[2, :, -500:] = torch.randn((Hkv, 500, d), generator=gen, device="cuda").bfloat16()
    q = torch.randn((190, 8, d), generator=gen, device="cuda").bfloat16() + 2
    desc = eb.cache_desc(K, V, 8, 64)
    out = torch.zeros_like(q)
    eb.eta_prefill(desc, DENSE, q, K, V, ints([0, 130, 130, 190]), ints(lens), out, workspace(desc))
    # weights of the zero keys are exp(0) each: 2 M of them, with values of zero
    for r in (130, 189):
        p = T - 60 + r - 130
        S = torch.einsum("hgd,htd->hgt", q[r].double().view(4, 2, d), K[2, :, T - 500:p + 1].double()) / math.sqrt(d)
        w = torch.exp(S)
        want = torch.einsum("hgt,htd->hgd", w, V[2, :, T - 500:p + 1].double()) / (w.sum(-1, keepdim=True) + T - 500)
        mass = torch.einsum("hgt,htd->hgd", w, V[2, :, T - 500:p + 1].double().abs()) / (w.sum(-1, keepdim=True) + T - 500)
        # 2 M additions of about one in fp32, several partial sums of 2^13 or fewer tiles: 2^-24 times a few thousand at most
        assert ((out[r].double().view(4, 2, d) - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -10) * mass + 1e-9).all()
    assert torch.all(out[:130] == 0)


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own, split items in both: what either gives alone."""
    both = [make([300, 1, 45], [900, 3000, 0], 2, 4, 128, 64, True, seed=23), make([77, 1], [5000, 4000], 4, 2, 64, 32, False, seed=24)]
    want = [call(s, DENSE)[0] for s in both]
    streams = [torch.cuda.Stream() for _ in both]
    args = []
    for s in both:
        if s["paged"]:
            desc, pages = eb.paged_cache_desc(s["K"], s["V"], s["B"], s["Hq"], t_cap=s["NB"] * s["b"]), eb.page_table(s["table"], s["K"].shape[0])
        else:
            desc, pages = eb.cache_desc(s["K"], s["V"], s["Hq"], s["b"]), None
        args.append((desc, pages, ints(s["starts"]), ints(s["lens"]), workspace(desc), [torch.full_like(s["q"], CANARY) for _ in range(10)]))
    torch.cuda.synchronize()
    for k in range(10):
        for s, stream, (desc, pages, starts, lens, ws, outs) in zip(both, streams, args):
            with torch.cuda.stream(stream):
                eb.eta_prefill(desc, DENSE, s["q"], s["K"], s["V"], starts, lens, outs[k], ws, pages=pages)
    torch.cuda.synchronize()
    for w, a in zip(want, args):
        assert all(torch.equal(w, x) for x in a[-1])
