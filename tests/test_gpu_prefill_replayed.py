"""One captured call of prompt attention, replayed over steps of other lengths: how work is shared out, split or whole, is decided on the device each time."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_prefill import CANARY, DENSE, ints, workspace

pytestmark = pytest.mark.gpu

ROWS = 640
STEPS = [                                   # new tokens, lengths, granted
    ([600, 0, 0, 0], [600, 0, 0, 0], [600, 0, 0, 0]),
    ([1, 1, 1, 1], [2000, 5, 1023, 1], [1, 1, 1, 1]),
    ([0, 0, 0, 0], [700, 3, 9, 1], [0, 0, 0, 0]),
    ([200, 1, 77, 300], [2048, 900, 77, 1500], [200, 1, 0, 300]),
    ([500, 100, 1, 30], [40, 100, 0, 5000], [500, 100, 1, 30]),
]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("paged,t_cap,d", [(True, 2048, 64), (False, 2048, 128), (False, 512, 64)])
def test_other_lengths_every_time(gated, paged, t_cap, d):
    gen = torch.Generator(device="cuda").manual_seed(121)
    B, Hkv, Hq, b = 4, 2, 8, 64
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    NB = t_cap // b
    if paged:
        K, V = randn(B * NB, Hkv, b, d), randn(B * NB, Hkv, b, d)
        table = torch.randperm(B * NB, generator=gen, device="cuda").int().view(B, NB)
        desc, pages = eb.paged_cache_desc(K, V, B, Hq, t_cap=t_cap), eb.page_table(table, B * NB)
    else:
        K, V = randn(B, Hkv, t_cap, d), randn(B, Hkv, t_cap, d)
        desc, pages = eb.cache_desc(K, V, Hq, b), None
    q, tau = randn(ROWS, Hq, d), torch.randn((ROWS, Hq), generator=gen, device="cuda")
    params, kw = (eb.DecodeParams(), dict(tau=tau)) if gated else (DENSE, {})
    start, lens, granted, status = ints([0] * 5), ints([0] * 4), ints([0] * 4), ints([0])
    ws, out = workspace(desc), torch.zeros_like(q)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        eb.eta_prefill(desc, params, q, K, V, start, lens, out, ws, granted=granted, status=status, pages=pages, **kw)
    for new, length, got in STEPS + STEPS[::-1]:
        starts = [sum(new[:i]) for i in range(5)]
        starts[4] = min(starts[4], ROWS)
        for t, v in ((start, starts), (lens, length), (granted, got), (status, [0])):
            t.copy_(ints(v))
        out.fill_(CANARY)
        graph.replay()
        torch.cuda.synchronize()
        want, flags = torch.full_like(out, CANARY), ints([0])
        eb.eta_prefill(desc, params, q, K, V, start.clone(), lens.clone(), want, workspace(desc), granted=granted.clone(), status=flags, pages=pages, **kw)
        assert torch.equal(out, want) and int(status) == int(flags)
        rows = torch.zeros(ROWS, dtype=torch.bool, device="cuda")
        for i in range(4):
            rows[starts[i]:min(ROWS, starts[i] + got[i])] = True
        assert torch.all(out[~rows] == CANARY) and torch.isfinite(out.float()).all()
