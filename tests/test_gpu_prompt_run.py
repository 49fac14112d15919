"""Prompts, forks and what follows, as a serving program makes the calls: pages planned, prompts written and attended, indexed, forked, decoded on by
all, one let go, the pool compacted, and one more step, eagerly and captured."""
import math

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from prefill_reference import reference

pytestmark = pytest.mark.gpu

B, HKV, G, D, BLOCK, T_CAP, PAGES = 6, 2, 4, 64, 32, 640, 90
HQ = HKV * G
LAYERS = 2


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def scratch(n):
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    return ws[-ws.data_ptr() % 256:][:n]


class Program:
    def __init__(self):
        self.gen = torch.Generator(device="cuda").manual_seed(5)
        randn = lambda *s: torch.randn(s, generator=self.gen, device="cuda")  # noqa: E731
        self.lens, self.n_free, self.status = ints([0] * B), ints([PAGES]), ints([0])
        self.table, self.free = ints([[0] * (T_CAP // BLOCK)] * B), torch.randperm(PAGES, generator=self.gen, device="cuda").int()
        self.shared = ints([0] * PAGES)
        # a pool of K and one of V per layer, as far as they are not written full of NaN
        self.K, self.V = ([torch.full((PAGES, HKV, BLOCK, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)] for _ in range(2))
        self.desc = eb.paged_cache_desc(self.K[0], self.V[0], B, HQ, t_cap=T_CAP)
        self.pages = eb.page_table(self.table, PAGES)
        self.index = [eb.alloc_summaries(self.desc, "cuda") for _ in range(LAYERS)]
        self.inv_freq = 10000.0 ** -(torch.arange(D // 2, dtype=torch.float64, device="cuda") / (D // 2))
        self.const = 0.4 * randn(HQ)
        self.prefill_ws, self.decode_ws = scratch(eb.eta_prefill_workspace_bytes(self.desc)), scratch(eb.eta_workspace_bytes(self.desc))
        self.pages_ws = scratch(eb.eta_pages_workspace_bytes(PAGES))
        self.randn = randn

    def buffers(self, rows):
        zeros = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        return dict(slots=zeros(rows, dtype=torch.int64), positions=zeros(rows), start=zeros(B + 1), granted=zeros(B),
                    q=zeros(LAYERS, rows, HQ, D, dtype=torch.bfloat16), out=zeros(LAYERS, rows, HQ, D, dtype=torch.bfloat16),
                    dense=zeros(LAYERS, rows, HQ, D, dtype=torch.bfloat16))

    def step(self, new, qkv, r, prompt):
        """New tokens into every layer's cache, attended, indexed."""
        eb.eta_plan_pages(BLOCK, T_CAP, new, self.lens, self.table, self.free, self.n_free, r["slots"], r["positions"], r["start"], r["granted"],
                          status=self.status)
        for layer in range(LAYERS):
            x, K, V, (musig, mnorm) = qkv[layer], self.K[layer], self.V[layer], self.index[layer]
            eb.eta_append_tokens(self.desc, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], r["slots"], r["positions"], r["q"][layer], K, V,
                                 inv_freq=self.inv_freq, paged=True, status=self.status)
            eb.eta_prefill(self.desc, eb.DecodeParams(beta=4.0), r["q"][layer], K, V, r["start"], self.lens, r["out"][layer], self.prefill_ws,
                           head_const=self.const, granted=r["granted"], status=self.status, pages=self.pages)
            eb.eta_prefill(self.desc, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), r["q"][layer], K, V, r["start"], self.lens, r["dense"][layer],
                           self.prefill_ws, granted=r["granted"], status=self.status, pages=self.pages)
            index = eb.eta_build_block_summaries_paged if prompt else eb.eta_append_summary_paged
            index(self.desc, self.pages, K, self.lens, musig, mnorm)

    def gathered(self, X, lens):
        return [X[self.table[i, :-(-n // BLOCK)].long()].transpose(0, 1).flatten(1, 2)[:, :n] for i, n in enumerate(lens)]

    def check(self, r):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        lens, start, granted = self.lens.tolist(), r["start"].tolist(), r["granted"].tolist()
        for layer in range(LAYERS):
            K, V = self.gathered(self.K[layer], lens), self.gathered(self.V[layer], lens)
            q = r["q"][layer]
            for out, te in ((r["out"][layer], self.const.expand(q.shape[0], -1)), (r["dense"][layer], None)):
                want, bound, counts = reference(q, K, V, start, lens, granted, 1 / math.sqrt(D), 4.0, te)
                assert ((out.double() - want).abs() <= bound)[counts].all() and torch.all(out[~counts] == 0)

    def decode(self, q, layer):
        """One query per sequence, dense."""
        out = torch.zeros((B, HQ, D), device="cuda")
        sel = torch.zeros((B, HKV, self.desc.nb_cap), dtype=torch.uint8, device="cuda")
        eb.eta_decode_paged(self.desc, self.pages, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), q, self.K[layer], self.V[layer], self.lens, *self.index[layer],
                            None, self.const, out, sel, self.decode_ws)
        return out

    def fork(self, parent, take):
        src, dst, got = ints([0] * B), ints([0] * B), ints([0] * B)
        eb.eta_fork_pages(BLOCK, T_CAP, parent, self.lens, self.table, self.shared, self.free, self.n_free, src, dst, got, take=take, status=self.status)
        eb.eta_copy_pages(self.K + self.V, src, dst, status=self.status)
        for musig, mnorm in self.index:
            eb.eta_fork_summaries(self.desc, parent, got, musig, mnorm, status=self.status)
        return got


def qkv(p, rows):
    return p.randn(LAYERS, rows, HQ + 2 * HKV, D).bfloat16()


@pytest.mark.parametrize("captured", [False, True])
def test_prompts_forks_and_what_follows(captured):
    p = Program()
    # two prompts, rows to spare
    r = p.buffers(520)
    new = ints([333, 0, 0, 150, 0, 0])
    p.step(new, qkv(p, 520), r, True)
    p.check(r)

    # three forks, one of a part of its parent; their index is what a build would write
    got = p.fork(ints([-1, 0, 0, -1, 3, -1]), ints([0, 999, 100, 0, 999, 0]))
    assert got.tolist() == [0, 333, 100, 0, 150, 0] and p.lens.tolist() == [333, 333, 100, 150, 150, 0]
    for layer in range(LAYERS):
        built = eb.alloc_summaries(p.desc, "cuda")
        eb.eta_build_block_summaries_paged(p.desc, p.pages, p.K[layer], p.lens, *built)
        for i, n in enumerate(p.lens.tolist()):
            for a, b in zip(built, p.index[layer]):
                assert torch.equal(a[i, :, :n // BLOCK], b[i, :, :n // BLOCK])

    # all of them go on by a token, beside the first chunk of another prompt
    r = p.buffers(80)
    new, x = ints([1, 1, 1, 1, 1, 70]), qkv(p, 80)
    if captured:
        state = [t.clone() for t in (p.lens, p.n_free, p.table, p.free)]
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            p.step(new, x, r, True)
        for _ in range(2):
            for t, was in zip((p.lens, p.n_free, p.table, p.free), state):
                t.copy_(was)
            graph.replay()
    else:
        p.step(new, x, r, True)
    p.check(r)
    assert p.lens.tolist() == [334, 334, 101, 151, 151, 70]

    # single tokens are what a dense decode step says, to the rounding of their outputs and weights
    last = r["start"][1:].long() - 1
    for layer in range(LAYERS):
        out = p.decode(r["q"][layer][last].contiguous(), layer)
        V = p.gathered(p.V[layer], p.lens.tolist())
        most = torch.tensor([v.abs().max().item() for v in V], device="cuda")[:, None, None]
        assert ((out - r["dense"][layer][last].float()).abs() <= 2 * 2.0 ** -8 * most).all()

    # a parent is let go: its children keep what they share; then the pool is compacted: the same bits from fewer pages
    before = [p.decode(r["q"][layer][last].contiguous(), layer) for layer in range(LAYERS)]
    free_before = int(p.n_free)
    eb.eta_free_pages(BLOCK, T_CAP, ints([1, 0, 0, 0, 0, 0]), p.lens, p.table, p.shared, p.free, p.n_free, p.pages_ws, status=p.status)
    assert int(p.n_free) == free_before + 1                # its last page, which was its own
    src, dst, n = ints([-1] * PAGES), ints([-1] * PAGES), ints([0])
    eb.eta_compact_pages(BLOCK, T_CAP, p.lens, p.table, p.shared, p.free, p.n_free, src, dst, n, p.pages_ws, status=p.status)
    eb.eta_copy_pages(p.K + p.V, src, dst, n_moves=n, status=p.status)
    live = PAGES - int(p.n_free)
    for i, m in enumerate(p.lens.tolist()):
        assert (p.table[i, :-(-m // BLOCK)] < live).all()
    for layer in range(LAYERS):
        after = p.decode(r["q"][layer][last].contiguous(), layer)
        assert torch.equal(after[1:], before[layer][1:]) and torch.all(after[0] == 0)
        for X in (p.K[layer], p.V[layer]):
            X[live:] = math.nan                            # nobody looks there any more

    # the place of the one that went is taken by a new prompt, the others go on
    r = p.buffers(300)
    p.step(ints([290, 1, 1, 1, 1, 1]), qkv(p, 300), r, True)
    p.check(r)
