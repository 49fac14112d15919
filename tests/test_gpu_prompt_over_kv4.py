"""Prompts over a 4-bit cache, the way that is built: new tokens written in 4 bits, the pool unpacked to bf16, attended there; forks of the 4-bit pages."""
import math

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from prefill_reference import reference
from test_gpu_page_sharing import ints
from test_gpu_prefill import CANARY, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,G,block", [(128, 4, 64), (64, 8, 32)])
@pytest.mark.parametrize("gated", [False, True])
def test_chunks_of_prompts_and_forks(d, G, block, gated):
    B, Hkv, t_cap, n_pages = 4, 2, 512, 60
    Hq = G * Hkv
    gen = torch.Generator(device="cuda").manual_seed(111)
    pool = torch.randint(0, 256, (n_pages, Hkv, eb.kv4_block_bytes(block, d)), generator=gen, device="cuda", dtype=torch.uint8)
    kdesc, kv4 = eb.kv4_cache_desc(pool, Hq, d, block, batch=B, t_cap=t_cap, k_scale=0.5, v_scale=0.25)
    K, V = (torch.zeros((n_pages, Hkv, block, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    desc = eb.paged_cache_desc(K, V, B, Hq, t_cap=t_cap)
    table = torch.full((B, t_cap // block), 2 ** 30, dtype=torch.int32, device="cuda")
    pages, ws = eb.page_table(table, n_pages), workspace(desc)
    lens, n_free, status, shared = ints([0] * B), ints([n_pages]), ints([0]), ints([0] * n_pages)
    free = torch.randperm(n_pages, generator=gen, device="cuda").int()
    params, const = (eb.DecodeParams(beta=3.0), 0.3 * torch.randn(Hq, generator=gen, device="cuda")) if gated else (eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), None)
    K0 = V0 = None
    for new in ([150, 0, 70, 0], [100, 0, 1, 0], [33, 40, 64, 0]):
        if new[1]:
            # sequence 1 begins as a copy of sequence 0; its last page is copied in 4 bits
            src, dst, got = ints([0] * B), ints([0] * B), ints([0] * B)
            eb.eta_fork_pages(block, t_cap, ints([-1, 0, -1, -1]), lens, table, shared, free, n_free, src, dst, got, status=status)
            eb.eta_copy_pages([pool], src, dst, status=status)
            assert got.tolist() == [0, 250, 0, 0]
        rows = sum(new) + 5
        x = torch.randn((rows, Hq + 2 * Hkv, d), generator=gen, device="cuda").bfloat16()
        slots, positions = torch.zeros(rows, dtype=torch.int64, device="cuda"), ints([0] * rows)
        start, granted = ints([0] * (B + 1)), ints([0] * B)
        q, out = torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.full((rows, Hq, d), CANARY, dtype=torch.bfloat16, device="cuda")
        eb.eta_plan_pages(block, t_cap, ints(new), lens, table, free, n_free, slots, positions, start, granted, status=status)
        eb.eta_append_tokens_kv4(kdesc, kv4, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, positions, q, pool, status=status)
        eb.eta_unpack_kv4(kdesc, kv4, pool, K, V)
        eb.eta_prefill(desc, params, q, K, V, start, lens, out, ws, head_const=const, granted=granted, status=status, pages=pages)
        assert int(status) == 0
        held = [[y[table[i, :-(-n // block)].long()].transpose(0, 1).flatten(1, 2)[:, :n] for i, n in enumerate(lens.tolist())] for y in (K, V)]
        want, bound, counts = reference(q, *held, start.tolist(), lens.tolist(), granted.tolist(), 1 / math.sqrt(d), 3.0,
                                        const.expand(rows, -1) if gated else None)
        assert ((out.double() - want).abs() <= bound)[counts].all() and torch.all(out[~counts] == CANARY) and counts.sum() == sum(new)
        if K0 is not None and new[1]:
            assert torch.equal(held[0][1][:, :250], K0) and torch.equal(held[1][1][:, :250], V0)
        K0, V0 = held[0][0].clone(), held[1][0].clone()
    assert lens.tolist() == [283, 290, 135, 0]
