"""The calls of a serving step together: pages planned from request lengths, new tokens normed, rotated and written, the index kept, thresholds
predicted, attention over the cache, 4-bit and bf16, with prompts, decoding, a finished request and a new one in its place; eagerly and as a
captured step.  Every step's attention is checked against the oracle on what the cache holds."""
import numpy as np
import pytest
import torch

from oracle import eta_oracle as orc
from tests import kv4_reference as ref
from tests.helpers import bits, compare_masks, heads_without_near_tie

pytestmark = pytest.mark.gpu

B, HKV, G, D, BLOCK, T_CAP, PAGES = 3, 2, 4, 64, 32, 512, 40
HQ = HKV * G


class Server:
    """What a program keeps: buffers sized once, tables and lengths on the device."""

    def __init__(self, four, seed=0):
        from paper_2609_20888_b200 import binding as eb
        self.eb, self.four = eb, four
        g = torch.Generator().manual_seed(seed)
        dev = lambda x: x.cuda()  # noqa: E731
        self.stride = T_CAP // BLOCK
        self.lens, self.n_free = torch.zeros(B, dtype=torch.int32).cuda(), torch.tensor([PAGES], dtype=torch.int32).cuda()
        self.table = torch.zeros((B, self.stride), dtype=torch.int32).cuda()
        self.free = dev(torch.randperm(PAGES, generator=g).int())
        self.status = torch.zeros(1, dtype=torch.int32).cuda()
        self.wq, self.wk = dev(1 + 0.2 * torch.randn((2, D), generator=g))
        self.inv_freq = (10000.0 ** -(torch.arange(D // 2, dtype=torch.float64) / (D // 2))).cuda()
        self.W = dev(torch.randn((HQ * D, HQ), generator=g) * 0.02)
        self.bias = dev(torch.full((HQ,), 0.5))
        if four:
            self.pool = torch.randint(0, 256, (PAGES, HKV, eb.kv4_block_bytes(BLOCK, D)), generator=g, dtype=torch.uint8).cuda()
            self.desc, self.kv4 = eb.kv4_cache_desc(self.pool, HQ, D, BLOCK, batch=B, t_cap=T_CAP, k_scale=0.5, v_scale=0.75)
            n = eb.eta_kv4_workspace_bytes(self.desc)
        else:
            self.K, self.V = (dev(torch.randn((PAGES, HKV, BLOCK, D), generator=g).to(torch.bfloat16)) for _ in range(2))
            self.desc = eb.paged_cache_desc(self.K, self.V, B, HQ, t_cap=T_CAP)
            n = eb.eta_workspace_bytes(self.desc)
        self.pages = eb.page_table(self.table, PAGES)
        self.musig, self.mnorm = eb.alloc_summaries(self.desc, "cuda")
        ws = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
        self.ws = ws[-ws.data_ptr() % 256:][:n]
        self.tau = torch.zeros((B, HQ), device="cuda")
        self.out = torch.zeros((B, HQ, D), device="cuda")
        self.sel = torch.zeros((B, HKV, self.desc.nb_cap), dtype=torch.uint8, device="cuda")

    def rows(self, n):
        return dict(slots=torch.zeros(n, dtype=torch.int64, device="cuda"), positions=torch.zeros(n, dtype=torch.int32, device="cuda"),
                    start=torch.zeros(B + 1, dtype=torch.int32, device="cuda"), granted=torch.zeros(B, dtype=torch.int32, device="cuda"),
                    q=torch.zeros((n, HQ, D), dtype=torch.bfloat16, device="cuda"))

    def append(self, new, qkv, r, release=None, prefill=False):
        """Plan, write, index.  qkv [rows, HQ + 2 HKV, D]"""
        eb = self.eb
        eb.eta_plan_pages(BLOCK, T_CAP, new, self.lens, self.table, self.free, self.n_free, r["slots"], r["positions"], r["start"], r["granted"],
                          release=release, status=self.status)
        parts = (qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], r["slots"], r["positions"], r["q"])
        how = dict(inv_freq=self.inv_freq, q_weight=self.wq, k_weight=self.wk, status=self.status)
        if self.four:
            eb.eta_append_tokens_kv4(self.desc, self.kv4, *parts, self.pool, **how)
            call = eb.eta_build_block_summaries_kv4 if prefill else eb.eta_append_summary_kv4
            call(self.desc, self.kv4, self.pool, self.lens, self.musig, self.mnorm, pages=self.pages)
        else:
            eb.eta_append_tokens(self.desc, *parts, self.K, self.V, paged=True, **how)
            call = eb.eta_build_block_summaries_paged if prefill else eb.eta_append_summary_paged
            call(self.desc, self.pages, self.K, self.lens, self.musig, self.mnorm)

    def attend(self, q):
        eb, p = self.eb, self.eb.DecodeParams(lwb=1)
        eb.eta_predict_threshold(q, self.W, self.bias, self.tau)
        if self.four:
            eb.eta_decode_kv4(self.desc, self.kv4, p, q, self.pool, self.lens, self.musig, self.mnorm, self.tau, None, self.out, self.sel, self.ws,
                              status=self.status, pages=self.pages)
        else:
            eb.eta_decode_paged(self.desc, self.pages, p, q, self.K, self.V, self.lens, self.musig, self.mnorm, self.tau, None, self.out, self.sel,
                                self.ws, status=self.status)

    def gathered(self):
        """The cache as bf16, sequence after sequence."""
        if self.four:
            K, V = (torch.empty((PAGES, HKV, BLOCK, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.eb.eta_unpack_kv4(self.desc, self.kv4, self.pool, K, V)
        else:
            K, V = self.K, self.V
        one = lambda X: X[self.table.long()].transpose(1, 2).reshape(B, HKV, T_CAP, D).cpu()  # noqa: E731
        return one(K), one(V)

    def check(self, q):
        torch.cuda.synchronize()
        assert self.status.item() & ~4 == 0
        K, V = self.gathered()
        lens = self.lens.cpu().numpy()
        for X in (K, V):                                    # what lies behind the sequences is not the oracle's to read
            for i, n in enumerate(lens):
                X[i, :, n:] = 0
        c = orc.Cache(bits(K), bits(V), lens.copy(), BLOCK)
        tau = self.tau.cpu().numpy()
        want = orc.decode_step(bits(q.cpu()), c, bits(self.musig.cpu()), self.mnorm.cpu().numpy(), tau=tau, lwb=1)
        sel = self.sel.cpu().numpy()
        for i, n in enumerate(lens):
            sel[i, :, n // BLOCK:] = 0
        near = compare_masks(sel, want["sel"], want["bound"], tau.astype(np.float64), lens, BLOCK, G, rescued=want["rescued"])
        keep = heads_without_near_tie(near, B, HQ)
        Kf, Vf = K.double().numpy(), V.double().numpy()
        tol = ref.output_bound(q.double().cpu().numpy(), Kf, Vf, 5.0, 1 / np.sqrt(D)) + (0 if self.four else 2.0 ** -14 * np.abs(Vf).max())
        assert np.abs(self.out.cpu().numpy() - want["out"])[keep].max() <= tol
        return want


def _tokens(g, n):
    return torch.randn((n, HQ + 2 * HKV, D), generator=g).to(torch.bfloat16).cuda()


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("four", [True, False])
def test_prompts_decoding_a_finished_request_and_a_new_one(four):
    g = torch.Generator().manual_seed(7)
    s = Server(four)
    r = s.rows(320)
    s.append(_ints([100, 33, 170]), _tokens(g, 320), r, prefill=True)          # 17 rows of padding
    torch.cuda.synchronize()
    assert s.lens.tolist() == [100, 33, 170] and s.n_free.item() == PAGES - 4 - 2 - 6 and r["slots"][303:].tolist() == [-1] * 17
    last = (r["start"][1:] - 1).long()
    s.attend(r["q"][last])
    s.check(r["q"][last])
    one = s.rows(B)
    for step in range(35):                                                    # across block borders of all three
        s.append(_ints([1] * B), _tokens(g, B), one)
        s.attend(one["q"])
        s.check(one["q"])
    # request 1 is over; another takes its place in the same call, beside two that go on
    held = [-(-n // BLOCK) for n in s.lens.tolist()]
    r = s.rows(90)
    s.append(_ints([1, 71, 1]), _tokens(g, 90), r, release=_ints([0, 1, 0]), prefill=True)
    torch.cuda.synchronize()
    assert s.lens.tolist() == [136, 71, 206]
    assert s.n_free.item() == PAGES - -(-136 // BLOCK) - 3 - -(-206 // BLOCK) and held[1] == 3
    used = [s.table[i, :-(-n // BLOCK)].tolist() for i, n in enumerate(s.lens.tolist())]
    assert len(set(sum(used, []))) == len(sum(used, [])) and not set(sum(used, [])) & set(s.free[:s.n_free.item()].tolist())
    last = (r["start"][1:] - 1).long()
    s.attend(r["q"][last])
    s.check(r["q"][last])


@pytest.mark.parametrize("four", [True, False])
def test_a_captured_step_does_what_eager_calls_do(four):
    """Two servers get the same tokens, one call by call, one from a graph that was captured once: equal bits, step after step."""
    g = torch.Generator().manual_seed(9)
    a, b = Server(four, 3), Server(four, 3)
    start = _tokens(g, 150)
    for s in (a, b):
        s.append(_ints([60, 31, 59]), start, s.rows(150), prefill=True)
    new, ra, rb = _ints([1] * B), a.rows(B), b.rows(B)
    qkv = torch.zeros((B, HQ + 2 * HKV, D), dtype=torch.bfloat16, device="cuda")
    # a first step eagerly on both, so that nothing is set up during the capture
    qkv.copy_(_tokens(g, B))
    for s, r in ((a, ra), (b, rb)):
        s.append(new, qkv, r)
        s.attend(r["q"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.append(new, qkv, rb)
        b.attend(rb["q"])
    for step in range(40):
        qkv.copy_(_tokens(g, B))
        a.append(new, qkv, ra)
        a.attend(ra["q"])
        graph.replay()
        torch.cuda.synchronize()
        for x in ("lens", "table", "free", "n_free", "tau", "musig", "mnorm", "sel", "out", "status"):
            assert torch.equal(getattr(a, x), getattr(b, x)), (step, x)
        assert torch.equal(ra["q"], rb["q"]) and torch.equal(a.pool, b.pool) if four else torch.equal(a.K, b.K)
    a.check(ra["q"])
