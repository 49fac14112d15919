"""eta_plan_pages against a plan made sequence by sequence in plain Python.  Whole numbers: everything has to be equal, what no one
names has to keep what it held."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def plan(block, t_cap, new, lens, table, free, n_free, n_rows, release=None):
    """The definition, one sequence after the other."""
    lens, table, free = list(lens), [list(r) for r in table], list(free)
    refused = False
    for i in range(len(lens)):
        if release is not None and release[i]:
            for j in range(-(-lens[i] // block)):
                free[n_free] = table[i][j]
                n_free += 1
            lens[i] = 0
    granted, row_start, slots, positions = [], [0], [-1] * n_rows, [0] * n_rows
    asked = 0
    available = n_free
    for i in range(len(lens)):
        want = max(0, new[i])
        row0 = row_start[-1]
        row_start.append(row0 + want)
        ok = lens[i] + want <= t_cap and row0 + want <= n_rows
        need = -(-(lens[i] + want) // block) - -(-lens[i] // block) if ok else 0
        asked += need
        ok = ok and (need == 0 or asked <= available)
        granted.append(want if ok else 0)
        refused = refused or granted[i] != want
        if not ok:
            continue
        held = -(-lens[i] // block)
        for j in range(need):
            n_free -= 1
            table[i][held + j] = free[n_free]
        for k in range(want):
            p = lens[i] + k
            slots[row0 + k], positions[row0 + k] = table[i][p // block] * block + p % block, p
        lens[i] += want
    return dict(seq_lens=lens, table=table, free=free, n_free=[n_free], slots=slots, positions=positions, row_start=row_start,
                granted=granted, status=[16 if refused else 0])


def state(block, stride, lens, n_pages, seed, spare=0):
    """Tables of sequences of the given lengths on scattered pages, and the stack of the others."""
    g = torch.Generator().manual_seed(seed)
    perm = torch.randperm(n_pages, generator=g).tolist()
    table, at = [], 0
    for n in lens:
        held = -(-n // block)
        table.append(perm[at:at + held] + [-7] * (stride - held))
        at += held
    assert at <= n_pages
    n_free = n_pages - at - spare
    return table, perm[at:at + n_free] + [-9] * (n_pages - n_free), n_free


def run(block, t_cap, new, lens, table, free, n_free, n_rows, release=None, in_place=False, wide=0):
    from paper_2609_20888_b200 import binding as eb
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    t = ints(table)
    if wide:                                     # rows of the table further apart than they are long
        t = torch.cat((t, torch.full((len(lens), wide), -5, dtype=torch.int32, device="cuda")), 1)[:, :t.shape[1]]
    d = dict(seq_lens=ints(lens), table=t, free=ints(free), n_free=ints([n_free]), row_start=ints([-3] * (len(lens) + 1)),
             slots=torch.full((n_rows,), -77, dtype=torch.int64, device="cuda"), positions=ints([-77] * n_rows), granted=ints([-3] * len(lens)),
             status=ints([0]))
    out = {} if in_place else {"seq_lens_out": torch.full_like(d["seq_lens"], -3), "n_free_out": torch.full_like(d["n_free"], -3)}
    eb.eta_plan_pages(block, t_cap, ints(new), d["seq_lens"], d["table"], d["free"], d["n_free"], d["slots"], d["positions"], d["row_start"],
                      d["granted"], release=None if release is None else ints(release), status=d["status"], **out)
    torch.cuda.synchronize()
    if not in_place:
        assert d["seq_lens"].tolist() == list(lens) and d["n_free"].tolist() == [n_free]
        d["seq_lens"], d["n_free"] = out["seq_lens_out"], out["n_free_out"]
    return {k: v.tolist() for k, v in d.items()}


def check(block, t_cap, new, lens, stride, n_pages, n_rows, release=None, seed=0, spare=0, **kw):
    table, free, n_free = state(block, stride, lens, n_pages, seed, spare)
    want = plan(block, t_cap, new, lens, table, free, n_free, n_rows, release)
    got = run(block, t_cap, new, lens, table, free, n_free, n_rows, release, **kw)
    for k in want:
        assert got[k] == want[k], k


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("in_place", [False, True])
def test_one_token_each_at_the_edges_of_blocks(block, in_place):
    lens = [0, 1, block - 1, block, block + 1, 2 * block - 1, 5 * block, 0]
    check(block, 8 * block, [1] * 8, lens, 8, 64, 8, in_place=in_place, wide=3)


@pytest.mark.parametrize("seed", range(6))
def test_prompts_releases_and_padded_rows(seed):
    g = torch.Generator().manual_seed(seed)
    B, block, stride = [1, 3, 37, 1024, 1025, 2500][seed], [64, 32, 128, 64, 32, 64][seed], 24
    r = lambda lo, hi: torch.randint(lo, hi, (B,), generator=g).tolist()  # noqa: E731
    lens = r(0, stride * block // 2)
    new = [n if c else 1 for n, c in zip(r(-3, 300), r(0, 3))]
    rows = sum(max(0, n) for n in new) + 13
    check(block, stride * block - 5, new, lens, stride, B * stride, rows, [int(c == 0) for c in r(0, 4)], seed, in_place=seed % 2 == 0)


def test_a_long_prompt_fills_many_pages_and_rows_take_a_kernel_of_their_own():
    check(32, 4096 * 32, [100000, 0, 1, 7000, -1, 5], [0, 17, 31, 100, 64, 0], 4096, 4000, 107100)


def test_rows_around_the_line_between_the_two_ways():
    for rows in (4095, 4096, 4097, 5120, 5121):
        check(64, 6400, [rows - 40, 0, 3, 30], [5, 6, 63, 0], 100, 200, rows, seed=rows)


def test_pages_run_out_in_order_and_who_needs_none_is_served():
    # two pages left: the first takes one, the second asks for three and gets none, the third needs none, the fourth would need one
    check(64, 1024, [10, 180, 5, 1, 0, 2], [64, 10, 20, 128, 64, 100], 16, 12, 198, spare=1)


def test_lengths_past_the_capacity_and_rows_past_the_buffer():
    check(64, 200, [1, 1, 50, 300, 7], [199, 200, 150, 0, 10], 4, 20, 359)
    check(64, 512, [8, 8, 8], [0, 0, 0], 8, 20, 20)          # the third's rows do not fit
    check(64, 512, [600, 8], [0, 0], 8, 20, 20)


def test_released_pages_are_on_top_of_the_stack_and_taken_again_at_once():
    check(32, 320, [64, 0, 33], [100, 64, 5], 10, 7, 97, release=[1, 1, 0])       # nothing but what came back
    check(32, 320, [0, 0, 0], [100, 0, 5], 10, 7, 0, release=[1, 1, 1])


def test_a_release_beyond_the_stack_is_cut_off():
    """The same pages handed back twice: the stack does not grow past its end, and the call says so."""
    block, lens = 32, [128, 64]
    table, free, n_free = state(block, 8, lens, 8, 3)
    got = run(block, 256, [0, 0], lens, table, free, 5, 0, release=[1, 1])
    assert got["n_free"] == [8] and got["status"] == [16] and got["free"] == free[:5] + table[0][:3] and got["seq_lens"] == [0, 0]


def test_captured_steps_go_on_from_one_another():
    """A step planned in place, captured once and replayed: every replay appends one token to every sequence."""
    from paper_2609_20888_b200 import binding as eb
    block, B, stride = 32, 5, 8
    lens = [0, 30, 31, 32, 63]
    table, free, n_free = state(block, stride, lens, B * stride, 1)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    d = dict(new=ints([1] * B), lens=ints(lens), table=ints(table), free=ints(free), n_free=ints([n_free]), pos=ints([0] * B),
             start=ints([0] * (B + 1)), got=ints([0] * B), slots=torch.zeros(B, dtype=torch.int64, device="cuda"))

    def call():
        eb.eta_plan_pages(block, stride * block, d["new"], d["lens"], d["table"], d["free"], d["n_free"], d["slots"], d["pos"], d["start"], d["got"])

    saved = {k: v.clone() for k, v in d.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k, v in saved.items():
        d[k].copy_(v)
    for _ in range(40):
        want = plan(block, stride * block, [1] * B, lens, table, free, n_free, B)
        graph.replay()
        torch.cuda.synchronize()
        lens, table, free, n_free = want["seq_lens"], want["table"], want["free"], want["n_free"][0]
        assert d["lens"].tolist() == lens and d["table"].tolist() == table and d["n_free"].tolist() == [n_free]
        assert d["slots"].tolist() == want["slots"] and d["pos"].tolist() == want["positions"]


def test_refusals_of_the_binding():
    from paper_2609_20888_b200 import binding as eb
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    slots = torch.zeros(4, dtype=torch.int64, device="cuda")
    table = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    ok = [64, 256, ints(2), ints(2), table, ints(8), ints(1), slots, ints(4), ints(3), ints(2)]
    eb.eta_plan_pages(*ok)
    for at, bad, what in [(2, ints(3), "seq_lens"), (3, ints(1), "seq_lens"), (4, table.t(), "block_table"), (1, 257, "block_table"),
                          (7, slots.int(), "slot_map"), (8, ints(3), "positions"), (9, ints(2), "row_start"), (10, ints(4)[::2], "granted"),
                          (6, ints(2), "n_free"), (5, ints(8).long(), "free_pages")]:
        args = list(ok)
        args[at] = bad
        with pytest.raises(eb.EtaError, match=what):
            eb.eta_plan_pages(*args)
