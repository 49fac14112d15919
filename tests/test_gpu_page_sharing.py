"""Forks, release, compaction and copies of pages against the same done sequence by sequence in plain Python.  Whole numbers and moved bytes:
everything has to be equal, what no one names has to keep what it held."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb

pytestmark = pytest.mark.gpu
REFUSED = eb.ETA_DEV_REFUSED


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def workspace(n_pages):
    n = eb.eta_pages_workspace_bytes(n_pages)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    return ws[-ws.data_ptr() % 256:][:n]


class Pool:
    """Tables, counts and stack as Python lists."""

    def __init__(self, block, stride, lens, n_pages, seed, parent=None):
        g = torch.Generator().manual_seed(seed)
        perm = torch.randperm(n_pages, generator=g).tolist()
        self.block, self.stride, self.n_pages, self.lens = block, stride, n_pages, list(lens)
        self.table, self.shared = [[-7] * stride for _ in lens], [0] * n_pages
        for i, n in enumerate(lens):
            u = parent[i] if parent else -1
            for j in range(-(-n // block)):
                if u >= 0 and j < n // block:
                    self.table[i][j] = self.table[u][j]
                    self.shared[self.table[u][j]] += 1
                else:
                    self.table[i][j] = perm.pop()
        self.n_free = len(perm)
        self.free = perm + [-9] * (n_pages - len(perm))

    def held(self, i):
        return min(-(-max(self.lens[i], 0) // self.block), self.stride)

    def tensors(self):
        return dict(lens=ints(self.lens), table=ints(self.table), shared=ints(self.shared), free=ints(self.free), n_free=ints([self.n_free]))

    def check(self, t):
        assert t["lens"].tolist() == self.lens
        assert t["table"].tolist() == self.table
        assert t["shared"].tolist() == self.shared
        assert t["free"].tolist() == self.free
        assert t["n_free"].tolist() == [self.n_free]


def fork(p, parent, take=None):
    src, dst, granted, refused = [-1] * len(parent), [-1] * len(parent), [0] * len(parent), False
    before, lens = p.n_free, list(p.lens)
    wanted = 0
    for i, u in enumerate(parent):
        if u < 0:
            continue
        if u >= len(parent) or u == i or lens[i] > 0 or parent[u] >= 0:
            refused = True
            continue
        T = max(0, min(lens[u], p.stride * p.block))
        if take is not None:
            T = min(T, max(0, take[i]))
        whole, tail = T // p.block, T % p.block != 0
        wanted += tail
        if tail and wanted > before:
            refused = True
            continue
        for j in range(whole):
            p.table[i][j] = p.table[u][j]
            p.shared[p.table[u][j]] += 1
        if tail:
            src[i], dst[i] = p.table[u][whole], p.free[before - wanted]
            p.table[i][whole] = dst[i]
            p.n_free -= 1
        granted[i] = p.lens[i] = T
    return src, dst, granted, refused


def release(p, which):
    count, refused = {}, False
    for i, r in enumerate(which):
        if r:
            for j in range(p.held(i)):
                page = p.table[i][j]
                if 0 <= page < p.n_pages:
                    count[page] = count.get(page, 0) + 1
                else:
                    refused = True
            p.lens[i] = 0
    for page in sorted(count):
        if count[page] > p.shared[page] + 1:
            refused = True
        if count[page] > p.shared[page]:
            p.shared[page] = 0
            if p.n_free < p.n_pages:
                p.free[p.n_free] = page
                p.n_free += 1
            else:
                refused = True
        else:
            p.shared[page] -= count[page]
    return refused


def compact(p):
    stack = p.free[:p.n_free]
    free = {x for x in stack if 0 <= x < p.n_pages}
    refused = len(free) != p.n_free
    live = p.n_pages - len(free)
    dst = [x for x in range(live) if x in free]
    src = [x for x in range(live, p.n_pages) if x not in free]
    to = dict(zip(src, dst))
    for i in range(len(p.lens)):
        for j in range(p.held(i)):
            page = p.table[i][j]
            if not 0 <= page < p.n_pages or page in free:
                refused = True
            else:
                p.table[i][j] = to.get(page, page)
    held = [p.shared[x] for x in src]
    for s, d, h in zip(src, dst, held):
        p.shared[s], p.shared[d] = 0, h
    p.n_free = len(free)
    p.free[:p.n_free] = [p.n_pages - 1 - k for k in range(p.n_free)]
    return src, dst, refused


def outs(t, in_place, names=("lens", "shared", "n_free")):
    if in_place:
        return {n: None for n in names}
    return {n: torch.full_like(t[n], 77) for n in names}


def merge(t, o):
    return {**t, **{k: v for k, v in o.items() if v is not None}}


def run_fork(p, parent, take=None, in_place=True):
    t = p.tensors()
    o = outs(t, in_place)
    src, dst, granted, status = ints([55] * len(parent)), ints([55] * len(parent)), ints([55] * len(parent)), ints([0])
    eb.eta_fork_pages(p.block, p.stride * p.block, ints(parent), t["lens"], t["table"], t["shared"], t["free"], t["n_free"], src, dst, granted,
                      take=None if take is None else ints(take), seq_lens_out=o["lens"], shared_out=o["shared"], n_free_out=o["n_free"], status=status)
    want = fork(p, parent, take)
    assert (src.tolist(), dst.tolist(), granted.tolist()) == want[:3]
    assert int(status) == (REFUSED if want[3] else 0)
    p.check(merge(t, o))


def run_release(p, which, in_place=True):
    t = p.tensors()
    o, status = outs(t, in_place), ints([0])
    eb.eta_free_pages(p.block, p.stride * p.block, ints(which), t["lens"], t["table"], t["shared"], t["free"], t["n_free"], workspace(p.n_pages),
                      seq_lens_out=o["lens"], shared_out=o["shared"], n_free_out=o["n_free"], status=status)
    assert int(status) == (REFUSED if release(p, which) else 0)
    p.check(merge(t, o))


def run_compact(p, in_place=True):
    t = p.tensors()
    o, status = outs(t, in_place, ("table", "shared", "n_free", "free")), ints([0])
    if not in_place:
        o["free"].copy_(t["free"])                     # (entries behind the stack are left as they are)
    src, dst, n = ints([55] * p.n_pages), ints([55] * p.n_pages), ints([55])
    eb.eta_compact_pages(p.block, p.stride * p.block, t["lens"], t["table"], t["shared"], t["free"], t["n_free"], src, dst, n, workspace(p.n_pages),
                         block_table_out=o["table"], shared_out=o["shared"], free_pages_out=o["free"], n_free_out=o["n_free"], status=status)
    want_src, want_dst, refused = compact(p)
    assert int(n) == len(want_src) and int(status) == (REFUSED if refused else 0)
    assert src.tolist() == want_src + [55] * (p.n_pages - len(want_src)) and dst.tolist() == want_dst + [55] * (p.n_pages - len(want_dst))
    p.check(merge(t, o))
    return src, dst, n


# small: one CTA; large: a cluster
SIZES = {"one page": (32, 1, [5, 0], 3), "small": (64, 6, [130, 64, 1, 0, 0, 384, 0, 200], 40), "bits": (32, 40, [1000, 0, 0, 1280, 7, 0], 97),
         "large": (64, 150, [9000, 0, 4096, 0, 0, 9600, 1, 0, 63, 0] * 6, 4001), "wide": (128, 3000, [300000, 0, 384000, 0], 9000)}


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("taken", [False, True])
def test_fork_then_release_then_compact(size, in_place, taken):
    block, stride, lens, n_pages = SIZES[size]
    p = Pool(block, stride, lens, n_pages, seed=1)
    whole = [i for i, n in enumerate(lens) if n > 0]
    parent = [whole[(3 * i) % len(whole)] if n == 0 else -1 for i, n in enumerate(lens)]
    take = [(i * 977) % (stride * block) for i in range(len(lens))] if taken else None
    run_fork(p, parent, take, in_place)
    run_release(p, [int(i % 3 == 0) for i in range(len(lens))], in_place)
    run_compact(p, in_place)
    run_compact(p, in_place)                              # nothing left to move
    run_release(p, [1] * len(lens), in_place)
    assert p.n_free == n_pages and not any(p.shared)
    run_compact(p, in_place)


def test_children_without_a_page_share_nothing():
    p = Pool(64, 4, [100, 0, 0, 128, 0, 0], 6, seed=2)      # two pages are free, three children want one
    run_fork(p, [-1, 0, 0, -1, 0, 3])
    assert p.lens == [100, 100, 100, 128, 0, 128]


def test_what_cannot_be_a_fork():
    p = Pool(64, 4, [100, 0, 0, 30, 0, 0, 0], 20, seed=3)
    # a place that is not empty, a parent out of range, a parent that is a child, itself, and one that can
    run_fork(p, [-1, 0, 7, 0, 1, 5, -1])


@pytest.mark.parametrize("take", [[0] * 4, [-5] * 4, [1] * 4, [64] * 4, [65] * 4, [10 ** 9] * 4])
def test_what_is_taken(take):
    run_fork(Pool(64, 5, [300, 0, 0, 0], 30, seed=4), [-1, 0, 0, 0], take)


def test_one_sequence_of_1024():
    p = Pool(32, 2, [40] + [0] * 1023, 1100, seed=5)
    run_fork(p, [-1] + [0] * 1023)
    run_release(p, [1] + [i % 2 for i in range(1023)])
    run_compact(p)


def test_numbers_outside_the_pool_are_skipped():
    p = Pool(64, 4, [256, 200, 0], 12, seed=6)
    p.table[0][1], p.table[1][2] = 12, -3
    run_release(p, [1, 1, 1])
    p = Pool(64, 4, [256, 200, 0], 12, seed=6)
    p.table[0][1] = 1 << 30
    p.free[0] = 99
    t = p.tensors()
    run_compact(p)
    assert p.table[0][1] == 1 << 30 and t is not None


def test_a_page_that_is_let_go_too_often_goes_back_once():
    p = Pool(64, 4, [256, 256], 12, seed=7)
    p.table[1] = list(p.table[0])                         # shared, but nobody counted
    run_release(p, [1, 1])
    assert p.free[:p.n_free].count(p.table[0][0]) == 1


def test_a_length_past_the_capacity():
    p = Pool(64, 3, [190, 0], 9, seed=8)
    p.lens[0] = 10000
    run_fork(p, [-1, 0])
    assert p.lens[1] == 192
    run_release(p, [1, 1])


def test_a_stack_that_holds_a_page_twice():
    p = Pool(64, 3, [100, 50], 9, seed=9)
    p.free[1] = p.free[0]
    run_compact(p)


@pytest.mark.parametrize("n_free", [-4, 0])
def test_an_empty_stack(n_free):
    p = Pool(64, 2, [128, 0, 128], 4, seed=10)
    t = p.tensors()
    t["n_free"].fill_(n_free)
    src, dst, granted, status = (ints([55] * 3) for _ in range(4))
    status = ints([0])
    eb.eta_fork_pages(64, 128, ints([-1, 0, -1]), t["lens"], t["table"], t["shared"], t["free"], t["n_free"], src, dst, granted, take=ints([0, 128, 0]),
                      status=status)
    assert granted.tolist() == [0, 128, 0] and int(status) == 0 and int(t["n_free"]) == 0


# ----------------------------------------------------------------------------------------------------------- copies

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.uint8, torch.float32])
@pytest.mark.parametrize("layout", ["pages", "heads first", "both in one", "one page run"])
def test_copies(dtype, layout):
    g = torch.Generator(device="cuda").manual_seed(1)
    pages, H, b, d = 37, 3, 32, 64
    make = lambda *s: torch.randint(0, 100, s, generator=g, device="cuda").to(dtype)  # noqa: E731
    if layout == "pages":
        pools = [make(pages, H, b, d), make(pages, H, b, d)]
    elif layout == "heads first":
        pools = [make(H, pages, b, d).transpose(0, 1), make(pages, b, H, d).transpose(1, 2)]
    elif layout == "both in one":
        kv = make(pages, 2, H, b, d)
        pools = [kv[:, 0], kv[:, 1]]
    else:
        pools = [make(pages, 9 * 16), make(pages, H, b, d)]
    src, dst = [3, -1, 7, 20, 5, 36], [4, 9, -1, 0, 21, 35]
    want = [x.clone() for x in pools]
    for w, x in zip(want, pools):
        for s, t in zip(src, dst):
            if s >= 0 and t >= 0:
                w[t] = x[s]
    status = ints([0])
    eb.eta_copy_pages(pools, ints(src), ints(dst), status=status)
    for w, x in zip(want, pools):
        assert torch.equal(w, x)
    # only the first two pairs, then a count past the list, then none
    more = [x.clone() for x in pools]
    eb.eta_copy_pages(pools, ints([1, 2, 6]), ints([10, 11, 12]), n_moves=ints([2]))
    for w, x in zip(more, pools):
        w[10], w[11] = x[1], x[2]
        assert torch.equal(w, x)
    eb.eta_copy_pages(pools, ints([1, 2, 6]), ints([10, 11, 12]), n_moves=ints([-1]))
    eb.eta_copy_pages(pools, ints([6]), ints([12]), n_moves=ints([1000]))
    for w, x in zip(more, pools):
        w[12] = x[6]
        assert torch.equal(w, x)
    assert int(status) == 0
    eb.eta_copy_pages(pools, ints([1, pages]), ints([pages, 2]), status=status)
    for w, x in zip(more, pools):
        assert torch.equal(w, x)
    assert int(status) == eb.ETA_DEV_BAD_SLOT


def test_many_large_copies():
    g = torch.Generator(device="cuda").manual_seed(2)
    pools = [torch.randint(0, 1 << 30, (600, 70001 * 4), generator=g, device="cuda", dtype=torch.int32) for _ in range(2)]
    perm = torch.randperm(600, generator=g, device="cuda").int()
    want = [x.clone() for x in pools]
    for w, x in zip(want, pools):
        w[perm[300:].long()] = x[perm[:300].long()]
    eb.eta_copy_pages(pools, perm[:300], perm[300:])
    for w, x in zip(want, pools):
        assert torch.equal(w, x)


def test_a_pool_past_two_to_the_32_bytes():
    pool = torch.zeros((1 << 17) + 5, 40960, dtype=torch.uint8, device="cuda")
    pool[3] = 7
    eb.eta_copy_pages([pool], ints([3]), ints([(1 << 17) + 4]))
    assert (pool[-1] == 7).all() and int(pool[:, 0].sum()) == 14


def test_pools_that_cannot_be_described():
    x = torch.zeros((4, 3, 8, 64), device="cuda")
    s = ints([0])
    for bad in ([x[:, :, ::2, ::2]], [x, torch.zeros((5, 64), device="cuda")], [x.cpu()], [x[0, 0, 0]], [], [x[:, :, :, :3]]):
        with pytest.raises(eb.EtaError):
            eb.eta_copy_pages(bad, s, s)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("d,b,nb_cap", [(128, 64, 33), (64, 32, 400), (128, 128, 1)])
def test_summaries(packed, d, b, nb_cap):
    g = torch.Generator(device="cuda").manual_seed(3)
    B, H = 7, 3
    if packed:
        musig = torch.randint(0, 255, (B, H, nb_cap, 3 * d), generator=g, device="cuda", dtype=torch.uint8)
    else:
        musig = torch.randn((B, H, nb_cap, 2, d), generator=g, device="cuda").half()
    mnorm = torch.randn((B, H, nb_cap), generator=g, device="cuda")
    parent, granted = [-1, 0, 0, -1, 3, 3, -1], [0, nb_cap * b, b * (nb_cap // 2) + b - 1, 0, b - 1, b, 900]
    desc = eb.CacheDesc(B, H, H, d, b, nb_cap * b, nb_cap, 0, 0, 0, 0, 0, 0)
    wm, wn = musig.clone(), mnorm.clone()
    for i, u in enumerate(parent):
        if u >= 0:
            n = granted[i] // b
            wm[i, :, :n], wn[i, :, :n] = wm[u, :, :n], wn[u, :, :n]
    status = ints([0])
    eb.eta_fork_summaries(desc, ints(parent), ints(granted), musig, mnorm, status=status)
    assert torch.equal(musig, wm) and torch.equal(mnorm, wn) and int(status) == 0
    # a parent that is none: nothing is done, and said
    eb.eta_fork_summaries(desc, ints([7, -1, 2, -1, -1, -1, -1]), ints([b] * B), musig, mnorm, status=status)
    assert torch.equal(musig, wm) and torch.equal(mnorm, wn) and int(status) == REFUSED


def test_captured():
    """A fork with its copies, in a graph: the same as eager, every time."""
    p = Pool(64, 20, [1000, 0, 0, 700, 0, 0], 70, seed=11)
    pool = torch.randn((70, 2, 64, 64), device="cuda").bfloat16()
    t = p.tensors()
    o = outs(t, False)
    src, dst, granted, parent = ints([0] * 6), ints([0] * 6), ints([0] * 6), ints([-1, 0, 3, -1, 0, 3])
    ws = workspace(70)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = pool.clone()
    gone, free = ints([1, 0, 0, 0, 0, 0]), t["free"].clone()
    after = {k: torch.zeros_like(t[k]) for k in ("lens", "shared", "n_free")}
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        eb.eta_fork_pages(64, 1280, parent, t["lens"], t["table"], t["shared"], t["free"], t["n_free"], src, dst, granted, seq_lens_out=o["lens"],
                          shared_out=o["shared"], n_free_out=o["n_free"])
        eb.eta_copy_pages([pool], src, dst)
        eb.eta_free_pages(64, 1280, gone, o["lens"], t["table"], o["shared"], free, o["n_free"], ws, seq_lens_out=after["lens"],
                          shared_out=after["shared"], n_free_out=after["n_free"])
    want = fork(p, [-1, 0, 3, -1, 0, 3])
    release(p, [1, 0, 0, 0, 0, 0])
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (src.tolist(), dst.tolist(), granted.tolist()) == want[:3]
        assert after["lens"].tolist() == p.lens and after["shared"].tolist() == p.shared and after["n_free"].tolist() == [p.n_free]
        assert free.tolist()[:p.n_free] == p.free[:p.n_free]
    for s, d in zip(want[0], want[1]):
        if s >= 0:
            keep[d] = keep[s]
    assert torch.equal(pool, keep)
